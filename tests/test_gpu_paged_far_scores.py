"""hawk_paged_attn with scores of any finite size: millions to many billions, of either sign, far and near ones among the rows of one
item, against the plain 64-bit form in every kernel and launch shape.

Queries and keys are numbers of few bits such that every product is exact, and every sum of them a multiple of a step that
leaves 19 to 23 bits (fp32 holds 24): the scores are exact in fp32, and the only roundings left are the ones that the bounds of
test_gpu_paged_attn.py count beside the scores' own.  The argument of the exponential is then off by 2^-22 of itself: the
difference of two scores is exact where it counts, its scale is a rounded constant.

Two terms more in fp16.  Below 2^-14 its numbers lie 2^-24 apart, so a small result is rounded by up to 2^-25, not by h of itself
(one key takes all here, and its value may be a number like 2.4e-6).  A small probability is rounded by up to 2^-25 too, or by all
of itself when it becomes 0.  Probabilities are rounded relative to the row's shift, which is no larger than the row's maximum, so
they are at least what they are after the division by their sum: each is off by min(p_j, 2^-25) at most there, an output by
sum_j min(p_j, 2^-25) |v_j|."""
import numpy as np
import pytest
import torch

from oracle import paged
from tests._paged import Batch, f64, half_step
from tests.test_gpu_paged_attn import _binary_tree, _check, _compare, _run
from tests.test_gpu_paged_padding import SHAPES

pytestmark = pytest.mark.gpu


def _far(b, kind, sign=1, seed=0):
    """Fills b's queries and keys.  Scores before the scale: sign * 1.3 * 2^33 + 2^15 t for "ties" (t = 0), "shuffled",
    "rising" and "falling" (t in 0 .. 255, so that the best keys take all), 1.3 * 2^24 + 4 t, t in 0 .. 15, for "mixed", and
    1.3 * 2^11 + 4 t for "near", where one rounding of the shift is still small enough to be left alone.  Row i of a
    stream: all of it times 2^-4 (i mod 3)."""
    rng = np.random.default_rng(seed)
    small = kind in ("mixed", "near")
    q, k = torch.zeros(b.D), torch.zeros(b.D)
    q[:18] = 2.0 ** 15
    k[:16] = sign * 83 / 64 * 2.0 ** {"mixed": 5, "near": -8}.get(kind, 14)  # 16 products
    k[16] = 27 / 16 * 2.0 ** (-8 if small else 8)               # 216, 27 * 2^19
    k[17] = 0 if small else 5.0                                 # 5 * 2^15
    q[18] = 4.0 if small else 2.0 ** 15
    q = q.expand(b.T, b.H, b.D).clone()
    for s, n in enumerate(b.new):
        for i in range(n):
            q[int(b.row_begin[s]) + i] *= 2.0 ** (-4 * (i % 3))
    b.q = q.to(b.dt)
    assert (b.q.float() == q).all()
    for s, kv in enumerate(b.kv):
        if b.new[s] == 0:
            continue
        t = {"ties": np.zeros(kv), "rising": np.arange(kv) * 255 // kv, "falling": 255 - np.arange(kv) * 255 // kv,
             "shuffled": rng.integers(0, 256, kv), "mixed": rng.integers(0, 16, kv), "near": rng.integers(0, 16, kv)}[kind]
        for j in range(b.need[s]):
            rows = min(b.page, kv - j * b.page)
            x = k.expand(b.H_kv, rows, b.D).clone()
            x[:, :, 18] = torch.from_numpy(t[j * b.page:j * b.page + rows].astype(np.float32))
            page = b.k_pages[int(b.block_table[s, j])]
            page[:, :rows] = x.to(b.dt)
            assert (page[:, :rows].float() == x).all()
    return b


def _check_chain(b):
    """_check, in fp16 with the terms for small results and probabilities."""
    if b.dt != torch.float16:
        return _check(b)
    got, status = _run(b)
    assert status == 0
    scale = b.D ** -0.5
    q, kp, vp = f64(b.q), f64(b.k_pages), f64(b.v_pages)
    want, size = paged.paged_attn(q, kp, vp, b.block_table.numpy(), b.row_begin.numpy(), b.kv_len.numpy(), scale)
    small = np.zeros_like(want)
    group = b.H // b.H_kv
    for s, (n, kv) in enumerate(zip(b.new, b.kv)):
        r0, ids = int(b.row_begin[s]), b.block_table[s, :b.need[s]].numpy()
        if n == 0:
            continue
        hidden = np.arange(kv)[None, :] > kv - n + np.arange(n)[:, None]
        for h in range(b.H):
            keys, values = (x[ids, h // group].reshape(-1, b.D)[:kv] for x in (kp, vp))
            e = np.where(hidden, -np.inf, q[r0:r0 + n, h] @ keys.T * scale)
            p = np.exp(e - e.max(1, keepdims=True))
            small[r0:r0 + n, h] = 2.0 ** -25 + np.minimum(p / p.sum(1, keepdims=True), 2.0 ** -25) @ np.abs(values)
    owned = ~np.isnan(want[:, 0, 0])
    assert (got[~owned] == 7.0).all(), "rows of no stream were written"
    got, want, size, small = got[owned], want[owned], size[owned], small[owned]
    assert np.isfinite(got).all()
    h, err = half_step(b.dt), np.abs(got - want)
    assert (err <= h * np.abs(want) + (h + 2.0 ** -11) * size + small).all()
    assert np.linalg.norm(err) <= (2 * h + 2.0 ** -11) * np.linalg.norm(want) + np.linalg.norm(small)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind,sign", [("ties", 1), ("ties", -1), ("shuffled", 1), ("shuffled", -1), ("rising", 1), ("falling", -1),
                                       ("mixed", 1), ("mixed", -1), ("near", 1), ("near", -1)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_scores_of_any_size(shape, kind, sign, dtype):
    _, new, kv, H, H_kv, D = shape
    _check_chain(_far(Batch(new, kv, H, H_kv, D, 16, dtype, seed=92, back=3), kind, sign))


@pytest.mark.parametrize("kind", ["ties", "shuffled", "mixed"])
@pytest.mark.parametrize("n,kv,H,H_kv,D", [(22, 2000, 2, 2, 128), (40, 100, 20, 20, 64), (20, 500, 12, 2, 64), (3, 60, 4, 4, 64)])
def test_trees(n, kv, H, H_kv, D, kind):
    masks = _binary_tree(n)
    masks[n // 2] = 0  # a node that sees the prefix alone
    _check(_far(Batch([n, n // 2], [n + kv, n // 2 + kv], H, H_kv, D, 16, seed=93), kind), masks)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_beyond_what_a_shift_could_hold(shape):
    """The same in bf16 at scores of 1e30: one exponent's rounding would be past every type's range."""
    _, new, kv, H, H_kv, D = shape
    b = _far(Batch(new, kv, H, H_kv, D, 16, seed=94), "shuffled")
    b.q *= 2.0 ** 67
    assert torch.isfinite(b.q).all() and np.abs(f64(b.q)).max() == 2.0 ** 82
    _check(b)


@pytest.mark.parametrize("D", [64, 128])
def test_a_far_row_beside_ordinary_ones(D):
    """Rows of N(0, 1) under keys of N(0, 1), one row of the same stream a million times as large: the ordinary ones keep their
    bounds, the large one is finite and inside its values' range (its scores are rounded in steps far above 1)."""
    for n, kv in ((3, 300), (12, 3000), (50, 2500), (150, 400)):
        b = Batch([n, n], [kv, kv - 9], 4, 2, D, 16, seed=95)
        row, good = n // 2, b.q[n // 2].clone()
        b.q[row] = (good.float() * 2.0 ** 30).to(b.dt)
        got, status = _run(b)
        assert status == 0 and np.isfinite(got[row]).all()
        assert np.abs(got[row]).max() <= np.nanmax(np.abs(f64(b.v_pages))) * (1 + 2.0 ** -7)
        b.q[row] = good
        want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                      b.kv_len.numpy(), D ** -0.5)
        got[row] = want[row]
        _compare(got, want, size, b.dt)


def _keys(b, major, minor):
    """Keys of b such that key j of stream s scores (before the scale) 16 * 2^15 major(s, j) + 2^15 minor(s, j)."""
    q = torch.zeros(b.D)
    q[:16] = q[18] = 2.0 ** 15
    b.q = q.expand(b.T, b.H, b.D).to(b.dt)
    for s, kv in enumerate(b.kv):
        for j in range(b.need[s]):
            for row in range(min(b.page, kv - j * b.page)):
                k = torch.zeros(b.D)
                k[:16], k[18] = major(s, j * b.page + row), minor(s, j * b.page + row)
                b.k_pages[int(b.block_table[s, j]), :, row] = k.to(b.dt)
                assert (b.k_pages[int(b.block_table[s, j]), 0, row].float() == k).all()
    return b


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_from_far_to_near_and_back(shape, up):
    """The first half of a stream's keys score -4 * 10^9 and the second around 0 (weights of 1 to 2^-16 among them), or around 0 and
    then 4 * 10^9: shifts cross the bound between the two ways in the middle of an item.  (fp32 numbers next to 2^32 lie 2^9 apart:
    steps of 4 there would not be exact, those of 2^10 are.)"""
    _, new, kv, H, H_kv, D = shape
    b = Batch(new, kv, H, H_kv, D, 16, seed=102, back=3)
    rng = np.random.default_rng(9)
    t = rng.integers(-15, 1, max(kv) + 1)
    step = 2.0 ** -13  # 4 units of a score, 0.7 in the exponent

    def major(s, j):
        return (0.0 if j >= b.kv[s] // 2 else -2.0 ** 13) if up else (0.0 if j < b.kv[s] // 2 else 2.0 ** 13)

    _check(_keys(b, major, lambda s, j: float(t[j]) * step * (256 if major(s, j) else 1)))


@pytest.mark.parametrize("scale,magnitude", [(2.0 ** -18, 2.0 ** 12), (40.0, 2.0 ** 12), (1e-30, 2.0 ** 14), (3.0, 2.0 ** -11)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_scales(shape, scale, magnitude):
    """Other factors than D^-1/2: scores that are large before it and small behind, the other way round, and all alike behind it (where it
    does not matter that 2^33 + 2^8 t is not an fp32 number; the others are)."""
    import paper_2510_25739_b200 as hawk
    _, new, kv, H, H_kv, D = shape
    b = Batch(new, kv, H, H_kv, D, 16, seed=103, back=3)
    t = np.random.default_rng(10).integers(0, 32, max(kv) + 1)
    _keys(b, lambda s, j: magnitude, lambda s, j: float(t[j]) * 2.0 ** -7)
    d = b.cuda()
    out = torch.full((b.T, H * D), 7.0, dtype=b.dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    hawk.paged_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, b.max_new, b.max_kv, scale, out=out, dev_status=status)
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), scale)
    assert int(status.item()) == 0
    _compare(f64(out).reshape(b.T, H, D), want, size, b.dt)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,kv", [([5, 9], [3, 0]), ([20, 12, 5], [9, 2000, 1]), ([60, 41], [50, 2000]), ([130, 90], [100, 0])])
def test_rows_that_see_nothing_beside_far_ones(new, kv, D):
    """Fewer keys than rows: the first rows see none and give zeros, the others' scores are far."""
    b = _far(Batch(new, kv, 2, 2, D, 16, seed=104), "shuffled", -1)
    _check(b)
    got, _ = _run(b)
    for s, (n, l) in enumerate(zip(new, kv)):
        r0 = int(b.row_begin[s])
        assert (got[r0:r0 + max(0, n - l)] == 0).all()
