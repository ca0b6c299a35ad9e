"""hawk_sample against the plain 64-bit form: filters, guidance, settings for each row, ties, masks, odd sizes, long rows, strides, bad values."""
import numpy as np
import pytest
import torch

import paper_2510_25739_b200 as hawk
from oracle import serving
from paper_2510_25739_b200 import binding, build
from tests import _serving as sv

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _logits(R, V, dtype="fp32", std=2.5, seed=0, masked=0.01):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, V), generator=g) * std
    if masked:
        x[torch.rand((R, V), generator=g) < masked] = -INF
    return x.to(TYPES[dtype]).cuda(), torch.rand(R, generator=g).cuda()


def _check(logits, u, got=None, exempt=0.02, **kw):
    """Runs hawk_sample and compares: tokens equal but where a decision is nearer than the sums' errors, probabilities within their bound."""
    names = dict(v_begin="begin", v_end="end")
    plain = {names.get(k, k): (v.tolist() if torch.is_tensor(v) else v) for k, v in kw.items()}
    token, prob, probs, margin, z = sv.exact_sample(logits, u.tolist(), **plain)
    R, V = probs.shape
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    token_prob = torch.full((R,), NAN, device="cuda")
    out = torch.full((R, V), NAN, device="cuda")
    if got is None:
        got = hawk.sample(logits, u, token_prob=token_prob, probs=out, dev_status=status, **kw)
    near = margin < serving.weight_error(V, probs.max(1))
    assert near.mean() <= exempt
    ok = ~near
    assert np.array_equal(got.cpu().numpy()[ok], token[ok])
    p = out.double().cpu().numpy()
    assert (np.abs(p - probs)[ok] <= sv.prob_bound(probs, z)[ok]).all()
    at = np.maximum(token, 0)
    tp = token_prob.double().cpu().numpy()
    assert (np.abs(tp - prob)[ok] <= sv.prob_bound(prob, z[np.arange(R), at])[ok]).all()
    # alone: the same token without the other outputs
    assert torch.equal(hawk.sample(logits, u, **kw), got)
    return int(status.item())


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=50), dict(top_k=2000), dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.05),
            dict(temperature=0.0), dict(temperature=1.3, top_k=500, top_p=0.95, min_p=0.01), dict(top_k=100000, top_p=0.5),
            dict(temperature=0.01, top_p=0.99), dict(temperature=30.0, top_k=3), dict(top_p=0.999999), dict(top_p=0.0), dict(min_p=1.0),
            dict(top_k=-3, top_p=2.0, min_p=-1.0)]


@pytest.mark.parametrize("kw", SETTINGS, ids=str)
@pytest.mark.parametrize("V", [1, 2, 33, 1000, 16384])
def test_filters(V, kw):
    logits, u = _logits(6, V, seed=V)
    assert _check(logits, u, **kw) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [7, 4095, 8192, 30001, 50257])
def test_types_and_odd_sizes(V, dtype):
    """Rows of odd length start anywhere inside 16 bytes; in 16 bits many logits are equal."""
    logits, u = _logits(9, V, dtype, seed=V)
    assert _check(logits, u, top_k=300, top_p=0.9) == 0
    assert _check(logits, u, top_p=0.8, min_p=0.001) == 0


@pytest.mark.parametrize("V", [32768, 32769, 65536, 100003, 262144])
def test_rows_shared_by_blocks(V):
    logits, u = _logits(3, V, "bf16", seed=V)
    for kw in (dict(), dict(top_k=2000), dict(top_p=0.9), dict(top_k=700, top_p=0.8, min_p=0.001), dict(temperature=0.0), dict(top_k=1)):
        assert _check(logits, u, **kw) == 0


@pytest.mark.parametrize("rows", [1, 2, 37, 149, 300, 700])
def test_numbers_of_rows(rows):
    """The launch shapes by number of rows give the same tokens as each row alone."""
    logits, u = _logits(rows, 4097, seed=rows)
    kw = dict(top_k=200, top_p=0.93)
    got = hawk.sample(logits, u, **kw)
    for r in range(0, rows, max(1, rows // 7)):
        assert int(hawk.sample(logits[r:r + 1], u[r:r + 1], **kw)) == int(got[r])
    assert _check(logits[:20], u[:20], got=None, **kw) == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_guidance(dtype):
    x, u = _logits(10, 16384, dtype, seed=5)
    logits = torch.cat([x[:5], (0.9 * x[:5].float() + 0.1 * x[5:].float()).to(x.dtype)])
    for kw in (dict(cfg_scale=7.5, top_k=2000), dict(cfg_scale=0.0), dict(cfg_scale=1.0, top_p=0.9), dict(cfg_scale=-2.0, temperature=0.0)):
        assert _check(logits, u[:5], **kw) == 0


def test_settings_of_each_row():
    R = 40
    logits, u = _logits(2 * R, 5000, seed=6)
    r = np.random.RandomState(0)
    kw = dict(temperature=r.choice([0.0, 0.5, 1.0, 2.0], R), top_p=r.choice([0.1, 0.9, 1.0, 3.0], R), min_p=r.choice([0.0, 0.02, -1.0], R),
              cfg_scale=r.choice([1.0, 4.0], R))
    kw = {k: torch.tensor(v, dtype=torch.float32, device="cuda") for k, v in kw.items()}
    kw["top_k"] = torch.tensor(r.choice([-1, 0, 1, 7, 4999, 5000, 6000], R), dtype=torch.int32, device="cuda")
    assert _check(logits, u[:R], **kw) == 0


def test_a_range_of_ids():
    """The layout of a text and image vocabulary: ids of the range only, strides wider than the row, probabilities into a wider tensor."""
    wide = torch.full((8, 70000), 50.0, device="cuda")
    x, u = _logits(8, 8192, seed=7)
    wide[:, 4:8196] = x
    logits = wide[:, :65536]
    assert _check(logits, u, v_begin=4, v_end=8196, top_k=2000, top_p=0.95) == 0
    assert _check(logits, u, v_begin=4, v_end=5, top_k=2000) == 0
    out = torch.full((8, 70000), -3.0, device="cuda")
    hawk.sample(logits, u, v_begin=4, v_end=8196, probs=out[:, 1:65537])
    assert (out[:, 0] == -3).all() and (out[:, 65537:] == -3).all() and (out[:, 1:5] == 0).all() and (out[:, 8197:65537] == 0).all()
    assert torch.allclose(out[:, 5:8197].sum(1), torch.ones(8, device="cuda"), atol=1e-4)


def test_many_draws_from_one_row():
    logits, _ = _logits(1, 3001, seed=8)
    u = torch.linspace(0, 1, 501, device="cuda")[:500].contiguous()
    assert _check(logits.expand(500, 3001), u, top_p=0.9) == 0


@pytest.mark.parametrize("kind", ["equal", "two", "steps", "sorted", "down", "outlier", "far", "spread", "masked", "last", "blocks"])
@pytest.mark.parametrize("V", [6000, 40000])
def test_distributions_that_mislead_a_sample(V, kind):
    """Ties by the thousand, sorted rows, one id far above or below all others, next to all ids masked."""
    R = 4
    g = torch.Generator().manual_seed(9)
    x, at = torch.randn((R, V), generator=g), torch.arange(V)
    if kind == "equal":
        x = torch.full((R, V), 1.5)
    elif kind == "two":
        x = (x > 1.0).float()
    elif kind == "steps":
        x = (x * 3).round()
    elif kind == "sorted":
        x = x.sort(1).values
    elif kind == "down":
        x = x.sort(1, descending=True).values
    elif kind == "outlier":
        x[:, 17] = 40.0
    elif kind == "far":
        x[:, 100] = -1e30
    elif kind == "spread":
        x = -(2.0 ** (x * 20))
    elif kind == "masked":
        x[:, 3:] = -INF
    elif kind == "last":
        x = torch.full((R, V), -5.0) + (at == V - 1) * 30.0
    elif kind == "blocks":
        x = x + (at // (V // 7)) * 2.0
    x, u = x.cuda(), torch.tensor([0.0, 0.3, 0.7, 0.999], device="cuda")
    for kw in (dict(), dict(top_k=40), dict(top_k=2500), dict(top_p=0.5), dict(top_p=0.97), dict(top_k=900, top_p=0.9, min_p=0.01)):
        assert _check(x, u, exempt=0.25, **kw) == 0  # (u = 0 is next to the border below the first id that is kept)


def test_extreme_values():
    V = 5000
    x, u = _logits(6, V, seed=10)
    x[0] = x[0] * 1e37            # (the range of fp32)
    x[1] = x[1] * 1e-38           # numbers next to the smallest
    x[2] = x[2] * 1e-3 + 1e6      # far from 0, steps of 1/16
    x[3] = 0.0
    x[3, 5:9] = -0.0
    for kw in (dict(), dict(top_k=100), dict(top_p=0.9), dict(temperature=1e-30, top_p=0.9), dict(temperature=1e30, top_k=20),
               dict(temperature=1e-45), dict(temperature=3e38, top_p=0.5), dict(temperature=1e-6, top_k=10, min_p=0.1)):
        assert _check(x, u, exempt=0.2, **kw) == 0


def test_values_that_cannot_be_drawn():
    x, u = _logits(5, 3000, seed=11, masked=0)
    x[0, 7], x[1, 8], x[2, :], x[3, :-1] = NAN, INF, -INF, NAN
    assert _check(x, u, top_p=0.9) == binding.DEV_NONFINITE
    assert int(hawk.sample(x, u)[2]) == -1 and int(hawk.sample(x, u)[3]) == 2999
    pair = torch.cat([x, torch.zeros_like(x)])
    pair[5 + 4, :100] = -INF
    assert _check(pair, u, cfg_scale=0.0) == binding.DEV_NONFINITE  # whatever the scale
    clean, v = _logits(2, 100, seed=12, masked=0.5)
    assert _check(torch.cat([clean, clean]), v, cfg_scale=2.0) == 0   # -inf is a mask, no flag


def test_settings_that_are_no_numbers():
    x, u = _logits(4, 900, seed=13)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    T = torch.tensor([NAN, -1.0, INF, 1.0], device="cuda")
    got = hawk.sample(x, u, temperature=T, dev_status=status)
    assert int(status) == binding.DEV_BAD_SETTING and torch.equal(got, hawk.sample(x, u))
    for name in ("top_p", "min_p"):
        status.zero_()
        got = hawk.sample(x, u, dev_status=status, **{name: torch.full((4,), NAN, device="cuda")})
        assert int(status) == binding.DEV_BAD_SETTING and torch.equal(got, hawk.sample(x, u))


def test_random_numbers_out_of_range():
    x, u = _logits(4, 700, seed=14, masked=0)
    low, high = hawk.sample(x, torch.zeros(4, device="cuda")), hawk.sample(x, torch.full((4,), 1 - 2.0 ** -24, device="cuda"))
    assert torch.equal(hawk.sample(x, torch.full((4,), -3.0, device="cuda")), low) and torch.equal(hawk.sample(x, torch.full((4,), NAN, device="cuda")), low)
    assert torch.equal(hawk.sample(x, torch.full((4,), 1.0, device="cuda")), high) and torch.equal(hawk.sample(x, torch.full((4,), INF, device="cuda")), high)


def test_its_distribution_is_what_the_verification_reads():
    """probs goes into cfg_accept as q_probs: drafts drawn from the target's own distribution are all accepted."""
    B, K, V = 3, 4, 16384
    logits, u = _logits(2 * B * K, V, seed=15, masked=0)
    logits = logits.reshape(2 * B, K, V)
    q = torch.empty((B, K, V), device="cuda")
    draft = hawk.sample(logits.reshape(2 * B * K, V), u[:B * K], cfg_scale=3.0, top_k=2000, probs=q.reshape(B * K, V))
    n, _ = hawk.cfg_accept(logits, q, draft.reshape(B, K), torch.full((B, K), 0.9999, device="cuda"), torch.rand((B, K + 1), device="cuda"),
                           0, V, 3.0, 1.0, 2000)
    assert (n == K).all()


def test_captured_and_on_another_stream():
    x, u = _logits(64, 16384, seed=16)
    want = hawk.sample(x, u, top_p=0.9)
    token, side = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hawk.sample(x, u, top_p=0.9, token=token)
    side.synchronize()
    assert torch.equal(token, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hawk.sample(x, u, top_p=0.9, token=token)
    for seed in (17, 18):
        y, v = _logits(64, 16384, seed=seed)
        x.copy_(y)
        u.copy_(v)
        graph.replay()
        assert torch.equal(token, hawk.sample(y, v, top_p=0.9))


def test_no_index_leaves_its_array():
    lib = build.build_debug_variant()
    x, u = _logits(5, 30001, "bf16", seed=19)
    for kw in (dict(), dict(top_k=300, top_p=0.9, v_begin=3, v_end=29000), dict(temperature=0.0)):
        out, status = torch.zeros((5, 30001), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        want = hawk.sample(x, u, **kw)
        with binding.alternate_library(lib):
            got = hawk.sample(x, u, probs=out, dev_status=status, **kw)
        assert torch.equal(got, want) and int(status) == 0


def test_refusals_with_tensors():
    x, u = _logits(4, 100)
    with pytest.raises(ValueError, match="u: expected shape"):
        hawk.sample(x, u[:3])
    with pytest.raises(ValueError, match="cfg_scale"):
        hawk.sample(x[:3], u[:1], cfg_scale=2.0)
    with pytest.raises(TypeError, match="top_k: expected torch.int32"):
        hawk.sample(x, u, top_k=u)
    with pytest.raises(TypeError, match="logits"):
        hawk.sample(x.double(), u)
    with pytest.raises(ValueError, match="contiguous"):
        hawk.sample(x.t(), u)
    with pytest.raises(binding.HawkError):
        hawk.sample(x, u, temperature=-1.0)
    with pytest.raises(binding.HawkError):
        hawk.sample(x, u, v_begin=5, v_end=101)
    assert hawk.sample(x[:0], u[:0]).shape == (0,)


@pytest.mark.parametrize("rows, V", [(16, 8192), (17, 20000), (32, 50257), (33, 50257), (100, 32000), (150, 32000), (149, 8193), (150, 16384),
                                     (40, 100003)])
def test_launch_shapes(rows, V):
    """Every way that a call's rows are dealt out to blocks gives the tokens of each row alone."""
    logits, u = _logits(rows, V, "bf16", seed=rows)
    kw = dict(top_k=1500, top_p=0.95)
    probs, one = torch.full((rows, V), NAN, device="cuda"), torch.full((1, V), NAN, device="cuda")
    got = hawk.sample(logits, u, probs=probs, **kw)
    for r in (0, rows // 2, rows - 1):
        assert int(hawk.sample(logits[r:r + 1], u[r:r + 1], probs=one, **kw)) == int(got[r])
        assert torch.equal(one[0], probs[r])
    assert _check(logits[:8], u[:8], **kw) == 0


@pytest.mark.parametrize("kw", [dict(), dict(top_k=3), dict(top_p=0.999999), dict(min_p=1e-30), dict(top_k=2, top_p=0.5)], ids=str)
@pytest.mark.parametrize("V", [6, 5000, 50257])
@pytest.mark.parametrize("top, T", [(40, 1e-6), (300, 1e-5), (500, 1.4e-6), (100, 3.5e-7), (100, 1e-6), (-40, 1e-6), (64, 1e-6), (-2, 9e-9),
                                    (1e30, 1e22), (7, 1e-20), (7, 1e-45), (0, 1e-45), (-3e38, 1e-6)])
def test_temperatures_next_to_nothing_beside_the_maximum(top, T, V, kw):
    """A step of fp32 at the maximum is some temperatures: no id but the maximum has a weight, wherever it stands and whatever the number."""
    at, u = [0, V // 2, V - 1, 3], torch.tensor([0.0, -1.0, NAN, 1 - 2.0 ** -24, 0.5], device="cuda")
    x = torch.full((len(at), V), -INF)
    x[:, 1:] = min(0.0, 0.9 * top if top > 0 else 1.1 * top) if top else -1.0
    x[:, 4] = torch.tensor(0.5 * top if top > 0 else 1.05 * top if top else -0.5)
    for r, p in enumerate(at):
        x[r, p] = top
    x = x.cuda()
    one = torch.zeros_like(x)
    one[range(len(at)), at] = 1
    for number in u:
        prob, probs, status = torch.full((len(at),), NAN, device="cuda"), torch.full_like(x, NAN), torch.zeros(1, dtype=torch.int32, device="cuda")
        token = hawk.sample(x, number.expand(len(at)).contiguous(), temperature=T, token_prob=prob, probs=probs, dev_status=status, **kw)
        assert token.tolist() == at and (prob == 1).all() and torch.equal(probs, one) and int(status) == 0


@pytest.mark.parametrize("top, T", [(40, 1e-6), (300, 1e-5), (100, 1e-6), (-40, 1e-6), (500, 1e-5), (-300, 2e-5)])
def test_neighbours_of_the_maximum_at_low_temperatures(top, T):
    """Ids some steps of fp32 below the maximum among others far below: those of a weight of 2^-45 and more are drawn, no others."""
    V = 3000
    r, top32, T32 = np.random.RandomState(abs(top)), np.float32(top), np.float64(np.float32(T))
    x = np.full(V, np.float32(top - abs(top) / 2), np.float32)
    below = [top32]
    for _ in range(14):
        below.append(np.nextafter(below[-1], np.float32(-np.inf)))
    place = np.sort(r.choice(V, 15, replace=False))
    x[place] = r.permutation(below)
    w = np.exp((x.astype(np.float64) - np.float64(top32)) / T32)
    assert (np.abs(w * 2.0 ** 45 - 1) > 1e-3).all()
    w[w < 2.0 ** -45] = 0
    run = np.cumsum(w)
    u = [0.0, -2.0, NAN, 0.3, 0.9, 0.99]
    want = [int(np.searchsorted(run, (n if n > 0 else 0.0) * run[-1], side="right")) for n in u]
    bound = serving.weight_error(V, 1 / run[-1]) + 2.0 ** -24
    for n in u[3:]:
        assert np.abs(run / run[-1] - n).min() > bound
    logits = torch.from_numpy(x).cuda().expand(len(u), V)
    prob, probs = torch.full((len(u),), NAN, device="cuda"), torch.full((len(u), V), NAN, device="cuda")
    token = hawk.sample(logits, torch.tensor(u, device="cuda"), temperature=T, token_prob=prob, probs=probs)
    assert token.tolist() == want
    z = np.clip((x.astype(np.float64) - np.float64(top32)) / T32, -1e4, 0)
    p = w / run[-1]
    assert (np.abs(probs.double().cpu().numpy() - p) <= sv.prob_bound(p, z)).all()
    assert (np.abs(prob.double().cpu().numpy() - p[want]) <= sv.prob_bound(p[want], z[want])).all() and (prob > 0).all()


def test_rows_past_2_31_elements():
    """Logits and distributions whose offsets pass 32 bits."""
    stride, V = 1 << 30, 1001
    x, u = _logits(4, V, "bf16", seed=20)
    far = torch.empty(3 * stride + V, dtype=torch.bfloat16, device="cuda").as_strided((4, V), (stride, 1))
    far.copy_(x)
    out = torch.empty(3 * stride + V, dtype=torch.float32, device="cuda").as_strided((4, V), (stride, 1))
    probs, kw = torch.full((4, V), NAN, device="cuda"), dict(top_k=300, top_p=0.9)
    assert torch.equal(hawk.sample(far, u, probs=out, **kw), hawk.sample(x, u, probs=probs, **kw)) and torch.equal(out, probs)
    assert torch.equal(hawk.sample(far, u[:2], cfg_scale=3.0), hawk.sample(x, u[:2], cfg_scale=3.0))


@pytest.mark.parametrize("rows", [6, 160])
def test_guided_drafts_of_an_image_vocabulary(rows):
    """Drafts as this framework verifies them: guidance, top-k 2000, distributions over the image's ids inside a wider vocabulary."""
    V, begin, end = 65536, 4, 8196
    x, u = _logits(rows, V, "bf16", seed=21)
    logits = torch.cat([x, (0.9 * x.float() + 0.1 * x.roll(1, 0).float()).bfloat16()])
    probs = torch.full((rows, V), NAN, device="cuda")
    kw = dict(cfg_scale=3.0, top_k=2000, v_begin=begin, v_end=end)
    got = hawk.sample(logits, u, probs=probs, **kw)
    assert (probs[:, :begin] == 0).all() and (probs[:, end:] == 0).all()
    few = list(range(0, rows, max(1, rows // 6)))
    pair = torch.cat([logits[few], logits[[rows + r for r in few]]])
    assert _check(pair, u[few], **kw) == 0 and torch.equal(hawk.sample(pair, u[few], **kw), got[few])
