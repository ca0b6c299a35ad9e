"""The calls around the paged cache as a user can make them on a GPU: what the Python layer refuses, tensors with unusual strides,
the smallest and the widest batches, and the build with index checks between guard words."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_25739_b200 import binding, build
from tests._paged import Batch, f64
from tests.test_gpu_paged_attn import _check, _compare, _run

pytestmark = pytest.mark.gpu


def _attn_args(b, d, **kw):
    a = dict(q=d.q, k_pages=d.k_pages, v_pages=d.v_pages, block_table=d.block_table, row_begin=d.row_begin, kv_len=d.kv_len,
             max_new=b.max_new, max_kv=b.max_kv, sm_scale=0.125)
    a.update(kw)
    return a


def test_attention_refusals():
    b = Batch([2, 3], [40, 20], 4, 2, 64, 16, seed=70)
    d = b.cuda()
    out = torch.full((b.T, 256), 7.0, dtype=b.dt, device="cuda")

    def refused(error, match, **kw):
        with pytest.raises(error, match=match):
            binding.paged_attn(**_attn_args(b, d, **{"out": out, **kw}))

    refused(TypeError, "bfloat16 or torch.float16", q=d.q.float())
    refused(TypeError, "k_pages", k_pages=d.k_pages.half())
    refused(TypeError, "block_table", block_table=d.block_table.long())
    refused(TypeError, "expected a torch.Tensor", q=[1.0])
    refused(TypeError, "a tensor is needed", kv_len=None)
    refused(TypeError, "anc_mask", anc_mask=torch.ones(3, dtype=torch.int32, device="cuda"))
    refused(ValueError, "anc_mask", anc_mask=torch.ones(2, dtype=torch.int64, device="cuda"))
    refused(ValueError, "k_pages", k_pages=d.k_pages.cpu())
    refused(ValueError, "row_begin", row_begin=d.row_begin[:2])
    refused(ValueError, "v_pages", v_pages=d.v_pages[:, :1])
    refused(ValueError, "block_table: must be contiguous", block_table=torch.stack([d.block_table, d.block_table], 2)[..., 0])
    refused(ValueError, "head dimension must be contiguous", q=torch.stack([d.q, d.q], 3)[..., 0])
    refused(ValueError, "out", out=out[:3])
    refused(ValueError, "3 dimensions", q=d.q.reshape(b.T, -1))
    refused(ValueError, "dev_status", dev_status=torch.zeros(2, dtype=torch.int32, device="cuda"))
    refused(ValueError, "max_kv", max_kv=1 << 40)
    refused(binding.HawkError, "status", max_kv=10 ** 6)                       # more than the table holds
    refused(binding.HawkError, "status", sm_scale=-1.0)
    refused(binding.HawkError, "status", q=torch.cat([d.q, d.q], 2)[..., 4:68])  # rows that begin 8 bytes off
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    big = Batch([64], [4000], 4, 2, 64, 16, seed=71)
    e = big.cuda()
    need = binding.paged_attn_workspace_bytes(1, 64, 64, 4, 2, 64, 4000)
    assert need > 16
    with pytest.raises(binding.HawkError):
        binding.paged_attn(**_attn_args(big, e, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda")))


def test_rope_refusals():
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    table, pos = torch.zeros((5, 64), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def refused(error, match, *args, **kw):
        with pytest.raises(error, match=match):
            binding.qk_norm_rope(*args, **kw)

    refused(ValueError, "norm", q, None, None, None, norm="batch")
    refused(TypeError, "position", q, None, pos.long(), table)
    refused(TypeError, "a tensor is needed", q, None, None, table)
    refused(TypeError, "cos_sin", q, None, pos, table.bfloat16())
    refused(ValueError, "position", q, None, pos[:2], table)
    refused(ValueError, "q_weight", q, None, None, None, norm="rms", q_weight=w[:32])
    refused(ValueError, "k_weight", q, q, None, None, norm="rms", q_weight=w, k_weight=torch.ones((4, 64), dtype=w.dtype, device="cuda"))
    refused(TypeError, "q_weight", q, None, None, None, norm="rms", q_weight=w.float())
    refused(binding.HawkError, "status", q, None, None, None, norm="rms")             # no weight
    refused(binding.HawkError, "status", q, None, None, None, norm="rms", q_weight=w, eps=-1.0)
    refused(binding.HawkError, "status", q, None, pos, torch.zeros((5, 24), device="cuda"))
    refused(binding.HawkError, "status", q[..., :32], None, None, None)
    pages = torch.zeros((2, 4, 16, 64), dtype=torch.bfloat16, device="cuda")
    bt, rb, kv = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 2), (2,), (1,)))
    with pytest.raises(TypeError, match="k: a tensor"):
        binding.rope_append(q, None, q, None, None, pages, pages, bt, rb, kv)
    with pytest.raises(ValueError, match="v:"):
        binding.rope_append(None, q, q[:, :2], None, None, pages, pages, bt, rb, kv)
    with pytest.raises(ValueError, match="k_pages"):
        binding.rope_append(None, q, q, None, None, pages[:, :2], pages, bt, rb, kv)


@pytest.mark.parametrize("n,kv,D", [(1, 60, 64), (20, 200, 128), (40, 3000, 128), (64, 900, 64), (130, 300, 128)])
def test_queries_that_share_memory(n, kv, D):
    """Heads that are one head seen several times (a stride of 0), then rows that are one row."""
    b = Batch([n, n], [kv, n], 4, 2, D, 16, seed=72)
    for q in (b.q[:, :1].expand(-1, 4, -1), b.q[:1].expand(b.T, -1, -1)):
        b.q = q.contiguous()
        d = b.cuda()
        d.q = q.cuda()[:, :1].expand(-1, 4, -1) if q.stride(1) == 0 else q[:1].contiguous().cuda().expand(b.T, -1, -1)
        assert 0 in d.q.stride()
        _check(b, dev=d)


@pytest.mark.parametrize("D", [64, 128])
def test_nothing_in_the_cache(D):
    """max_kv 0: every row sees nothing; a batch without a row."""
    b = Batch([2, 0], [0, 0], 2, 2, D, 16, seed=73)
    got, status = _run(b)
    assert status == 0 and (got == 0).all()
    b = Batch([0, 0], [5, 9], 2, 2, D, 16, seed=74, front=3)
    got, status = _run(b, max_new=4, max_kv=16)
    assert status == 0 and (got == 7.0).all()


@pytest.mark.parametrize("S,H,D", [(4096, 32, 128), (4096, 64, 64), (3000, 20, 128)])
def test_wide_batches_of_grouped_heads(S, H, D):
    """The largest batch at up to 64 rows per kv head: the list of streams next to everything else in shared memory."""
    rng = np.random.default_rng(S + H)
    kv = [int(x) for x in rng.integers(1, 30, S)]
    _check(Batch([1] * S, kv, H, 1, D, 8, seed=75))


def test_keys_with_infinities_behind_the_last_one():
    """Page rows that nobody owns hold infinities instead of NaN."""
    _check(Batch([5, 40, 130], [130, 77, 300], 4, 2, 64, 16, seed=76, poison=float("inf")))
    _check(Batch([5, 40], [3000, 2077], 4, 2, 128, 16, seed=77, poison=float("inf")))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,kv,D", [(3, 70, 64), (20, 200, 64), (20, 200, 128), (16, 3000, 128), (50, 2000, 64), (150, 400, 128), (90, 3000, 64)])
def test_a_bad_query_row_stays_alone(n, kv, D, bad):
    """A query row of NaN or infinities spoils its own result and no other row's."""
    b = Batch([n, n], [kv, kv - 9], 4, 2, D, 16, seed=81)
    row = n // 2
    good = b.q[row].clone()
    b.q[row, 1] = bad
    got, status = _run(b)
    assert status == 0 and np.isnan(got[row, 1]).any()
    b.q[row] = good
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), D ** -0.5)
    got[row, 1] = want[row, 1]
    _compare(got, want, size, b.dt)


def test_graphs_that_share_a_workspace():
    """Two captured calls of different kernels in one workspace, replayed in turn on one stream."""
    bs = [Batch([40], [3000], 2, 2, 128, 16, seed=78), Batch([100, 3], [2000, 50], 2, 2, 64, 16, seed=79)]
    ds = [b.cuda() for b in bs]
    outs = [torch.zeros((b.T, b.H * b.D), dtype=b.dt, device="cuda") for b in bs]
    need = max(binding.paged_attn_workspace_bytes(b.S, b.T, b.max_new, b.H, b.H_kv, b.D, b.max_kv) for b in bs)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for b, d, o in zip(bs, ds, outs):
        args = _attn_args(b, d, out=o, workspace=ws, sm_scale=b.D ** -0.5)
        binding.paged_attn(**args)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.paged_attn(**args)
        graphs.append(g)
    for o in outs:
        o.zero_()
    for _ in range(5):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for b, o in zip(bs, outs):
        want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                      b.kv_len.numpy(), b.D ** -0.5)
        _compare(f64(o).reshape(b.T, b.H, b.D), want, size, b.dt)


@pytest.fixture(scope="module")
def debug_lib():
    return build.build_debug_variant()


@pytest.mark.parametrize("new,kv,H,H_kv,D,tree", [
    ([4] * 8, [300] * 8, 4, 4, 64, False),              # a block per item
    ([8] * 40, [200] * 40, 20, 20, 64, False),          # equal shares of warps
    ([60, 0, 41], [3000, 5, 2000], 2, 2, 128, False),   # equal shares of blocks
    ([22] * 3, [2422, 22, 500], 6, 2, 64, True),
    ([300, 1, 90], [400, 20, 90], 2, 2, 128, False),    # chunks
    ([100], [3000], 6, 2, 64, False),                   # split over the keys
])
def test_index_checks_and_guards(new, kv, H, H_kv, D, tree, debug_lib):
    """Rows in front and behind, with guard rows around `out`; every computed index inside its array."""
    b = Batch(new, kv, H, H_kv, D, 16, seed=80, front=2, back=3)
    d = b.cuda()
    full = torch.full((b.T + 64, H * D), 3.0, dtype=b.dt, device="cuda")
    out = full[32:32 + b.T]
    masks = torch.from_numpy(np.array([(2 << i) - 1 for i in range(max(new))], dtype=np.uint64).view(np.int64)).cuda() if tree else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.full((binding.paged_attn_workspace_bytes(b.S, b.T, b.max_new, H, H_kv, D, b.max_kv) + 4096,), 85, dtype=torch.uint8,
                    device="cuda")
    with binding.alternate_library(debug_lib):
        binding.paged_attn(**_attn_args(b, d, out=out, dev_status=status, anc_mask=masks, workspace=ws[:-4096], sm_scale=D ** -0.5))
        torch.cuda.synchronize()
    assert int(status.item()) == 0
    begin = b.row_begin.tolist()
    assert (full[:32 + begin[0]] == 3.0).all() and (full[32 + begin[-1]:] == 3.0).all() and (ws[-4096:] == 85).all()
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), D ** -0.5)
    got = f64(out).reshape(b.T, H, D)
    got[:begin[0]] = got[begin[-1]:] = 7.0
    _compare(got, want, size, b.dt)


def test_chunks_without_keys_again_and_again():
    """Chunks whose rows see nothing among chunks that do: blocks without work end while others of their SM begin."""
    rng = np.random.default_rng(82)
    new = [int(x) for x in rng.integers(65, 200, 120)]
    kv = [0 if s % 2 else n for s, n in enumerate(new)]
    for D in (64, 128):
        b = Batch(new, kv, 2, 2, D, 16, seed=83)
        d = b.cuda()
        first, status = _run(b, dev=d)
        assert status == 0
        for s in range(1, 120, 2):
            assert (first[int(b.row_begin[s]):int(b.row_begin[s + 1])] == 0).all()
        _check(b, dev=d)
        for _ in range(30):
            again, status = _run(b, dev=d)
            assert status == 0 and np.array_equal(first, again)


def test_what_the_device_finds_wrong_in_long_streams():
    """The same findings as in test_gpu_paged_attn.py, in the kernel for few long streams."""
    b = Batch([12, 9, 3], [3000, 2000, 500], 2, 2, 128, 16, seed=84)
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), 128 ** -0.5)

    def others_stand(got, s):
        ok = np.ones(b.T, dtype=bool)
        ok[int(b.row_begin[s]):int(b.row_begin[s + 1])] = False
        h = 2.0 ** -8
        assert (np.abs(got - want)[ok] <= (h * np.abs(want) + (h + 2.0 ** -11) * size)[ok]).all()

    for page in (b.n_pages, -1, 2 ** 31 - 1):
        d = b.cuda()
        d.block_table[1, 77] = page
        got, status = _run(b, dev=d)
        assert status == binding.DEV_BAD_PAGE
        others_stand(got, 1)
    for bad in (3001, -1):
        d = b.cuda()
        d.kv_len[2] = bad
        got, status = _run(b, dev=d)
        assert status == binding.DEV_BAD_PREFIX or (bad > 0 and status == binding.DEV_BAD_PREFIX | binding.DEV_BAD_PAGE)
        others_stand(got, 2)
    d = b.cuda()
    d.row_begin[1] = 30
    got, status = _run(b, dev=d)
    assert status == binding.DEV_BAD_ROWS and (got[:21] == 7.0).all()
    d = b.cuda()
    got, status = _run(b, dev=d, max_new=11)
    assert status == binding.DEV_BAD_ROWS and (got[:12] == 7.0).all()
    others_stand(got, 0)
