"""GPU parity of hawk_paged_attn against the plain 64-bit form.

Bounds.  Scores, sums and accumulators are fp32; what is rounded to the 16-bit type with half step h (bf16 2^-8, fp16 2^-11)
are the probabilities (each p_j by at most h p_j, which moves an output by at most h sum_j p_j |v_j| = h size) and the result
(h |want|).  The rest, per element relative to `size`: scores of D products in fp32 (at most D 2^-24 sum |q k| scale, with
sum |q k| scale below 32 for these inputs: 128 * 2^-24 * 32 = 2^-12), the exponential's argument and value (2^-19), the sums over the
keys (2^-12 covers 4096 additions).  Together: |got - want| <= h |want| + (h + 2^-11) size.
That bound holds whatever the signs of the roundings.  They are independent, so the whole output is much nearer: its
2-norm error is at most h sqrt(sum p^2 v^2) for the probabilities and h |want| for the result, and for centred values the
first root is no larger than |want| on average: ||got - want|| <= 2 h ||want|| + 2^-11 ||want||.  One key missed or
counted twice among thousands is more than that.
"""
import numpy as np
import pytest
import torch

from oracle import paged
from tests._paged import Batch, f64, half_step

pytestmark = pytest.mark.gpu


def _run(b, masks=None, dev=None, **kw):
    import paper_2510_25739_b200 as hawk
    d = b.cuda() if dev is None else dev
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((b.T, b.H * b.D), 7.0, dtype=b.dt, device="cuda")
    m = None if masks is None else torch.from_numpy(np.array(masks, dtype=np.uint64).view(np.int64)).cuda()
    r = hawk.paged_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, kw.get("max_new", b.max_new),
                        kw.get("max_kv", b.max_kv), b.D ** -0.5, anc_mask=m, out=out, dev_status=status)
    torch.cuda.synchronize()
    assert r is out
    return f64(out).reshape(b.T, b.H, b.D), int(status.item())


def _compare(got, want, size, dt):
    owned = ~np.isnan(want[:, 0, 0])
    assert (got[~owned] == 7.0).all(), "rows of no stream were written"
    got, want, size = got[owned], want[owned], size[owned]
    assert np.isfinite(got).all()
    h = half_step(dt)
    err = np.abs(got - want)
    bound = h * np.abs(want) + (h + 2.0 ** -11) * size
    assert (err <= bound).all(), (err.max(), np.unravel_index(np.argmax(err - bound), err.shape))
    assert np.linalg.norm(got - want) <= (2 * h + 2.0 ** -11) * np.linalg.norm(want)


def _check(b, masks=None, **kw):
    got, status = _run(b, masks, **kw)
    assert status == 0
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), b.D ** -0.5, masks)
    _compare(got, want, size, b.dt)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,H,H_kv,page", [(64, 4, 4, 16), (64, 6, 2, 32), (128, 4, 1, 16), (128, 2, 2, 24)])
def test_decode(dtype, D, H, H_kv, page):
    """One row a stream; keys from one to several hundred, pages that end inside a tile."""
    _check(Batch([1] * 7, [1, 7, 16, 17, 129, 300, 33], H, H_kv, D, page, dtype, seed=1))


@pytest.mark.parametrize("D,page", [(64, 16), (128, 8), (64, 256), (128, 64), (64, 40)])
def test_drafted_blocks(D, page):
    """A handful of rows a stream, uneven, one stream idle, rows of nobody in front and behind."""
    _check(Batch([5, 1, 0, 8, 3], [400, 1, 77, 8, 131], 6, 3, D, page, seed=2, front=2, back=3, packed=True))


@pytest.mark.parametrize("layout", ["hrd", "rhd", "kv"])
@pytest.mark.parametrize("D", [64, 128])
def test_layouts(layout, D):
    _check(Batch([4, 2, 150], [90, 65, 200], 4, 2, D, 16, seed=3, layout=layout, packed=True))


@pytest.mark.parametrize("S,n,kv,H,H_kv,D", [
    (16, 5, 300, 20, 20, 64),    # 320 items of one column tile: merged inside the block
    (12, 6, 260, 32, 32, 128),   # the same at D = 128
    (2, 4, 100, 16, 16, 64),     # short items: one warp each
    (40, 8, 200, 20, 20, 64),    # equal shares and a merge kernel
    (3, 2, 2100, 8, 1, 64),      # eight heads share the keys, long items cut into many shares
    (2, 1, 4000, 2, 2, 128),
])
def test_launch_shapes(S, n, kv, H, H_kv, D):
    """Every launch shape of the few-rows kernel; uneven keys inside each."""
    rng = np.random.default_rng(S + kv)
    kvs = [int(x) for x in rng.integers(n, kv + 1, S)]
    kvs[0] = kv
    _check(Batch([n] * S, kvs, H, H_kv, D, 16, seed=4))


@pytest.mark.parametrize("rows", [(8, 8), (16, 9), (24, 17), (32, 25), (33, 40), (64, 48)])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_up_to_the_chunk_kernel(rows, D):
    """Row counts around every column-tile count of the few-rows kernel, cut into several items where they do not fit one."""
    _check(Batch(list(rows), [300, 111], 2, 2, D, 16, seed=5))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,kv", [(65, 65), (127, 400), (128, 128), (129, 1000), (256, 300), (257, 257), (300, 777)])
def test_chunks(dtype, D, n, kv):
    """Chunks of many rows, alone: with and without a prefix, one query tile and several, last tiles of every fill."""
    _check(Batch([n], [kv], 2, 1, D, 16, dtype, seed=6))


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8])
def test_chunk_groups(G):
    """Query heads per kv head that do and do not divide a tile's 128 rows."""
    _check(Batch([90, 130], [250, 130], 2 * G, 2, 64, 32, seed=7))


@pytest.mark.parametrize("page", [8, 24, 48, 128, 256])
def test_chunk_pages(page):
    _check(Batch([150, 100], [500, 331], 2, 2, 128, page, seed=8))


@pytest.mark.parametrize("D", [64, 128])
def test_chunk_split_over_the_keys(D):
    """Few query tiles over many keys: the key range is split over blocks and joined."""
    _check(Batch([70, 100], [2500, 1203], 2, 2, D, 16, seed=9))


def test_mixed_batch():
    """Decode steps, drafted blocks, an idle stream and chunks in one call."""
    _check(Batch([1, 200, 5, 0, 70, 1], [600, 350, 17, 9, 1100, 1], 4, 2, 64, 16, seed=10, front=1, back=2, packed=True))


def test_many_blocks():
    """More blocks than the GPU has SMs, every query tile count."""
    rng = np.random.default_rng(3)
    new = [int(x) for x in rng.integers(60, 400, 9)]
    kv = [n + int(x) for n, x in zip(new, rng.integers(0, 200, 9))]
    _check(Batch(new, kv, 8, 8, 64, 16, seed=11))


@pytest.mark.parametrize("new,kv", [
    ([3, 2], [1, 0]),          # fewer keys than rows: the first rows see nothing; no keys at all
    ([5, 5], [5, 0]),
    ([130, 90], [100, 0]),     # the same in the chunk kernel
    ([200, 1], [1, 1]),
])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_see_nothing(new, kv, D):
    b = Batch(new, kv, 2, 2, D, 16, seed=12)
    _check(b)
    got, _ = _run(b)
    for s, (n, l) in enumerate(zip(new, kv)):
        r0 = int(b.row_begin[s])
        assert (got[r0:r0 + max(0, n - l)] == 0).all()


def _binary_tree(n):
    masks = []
    for i in range(n):
        masks.append((masks[(i - 1) // 2] if i else 0) | 1 << i)
    return masks


@pytest.mark.parametrize("n,H,H_kv,D,dtype", [(3, 2, 2, 64, "bf16"), (22, 4, 4, 128, "fp16"), (31, 4, 2, 64, "bf16"),
                                              (63, 4, 1, 64, "bf16"), (64, 2, 2, 128, "bf16"), (40, 8, 1, 128, "fp16")])
def test_trees(n, H, H_kv, D, dtype):
    """Candidate trees; streams that bring only the first nodes of the tree ride along."""
    _check(Batch([n, n, max(1, n // 2)], [n + 333, n, n + 40], H, H_kv, D, 16, dtype, seed=13), _binary_tree(n))


def test_tree_rows_without_any_key():
    masks = [0, 2, 0, 8]  # nodes 0 and 2 do not even see themselves
    b = Batch([4, 4], [4, 30], 2, 2, 64, 16, seed=14)
    _check(b, masks)
    got, _ = _run(b, masks)
    assert (got[0] == 0).all() and (got[2] == 0).all() and (got[1] != 0).any()


def test_chain_mask_equals_the_chain_bit_for_bit():
    b = Batch([7, 5], [300, 41], 4, 2, 64, 16, seed=15)
    got1, _ = _run(b)
    got2, _ = _run(b, [(2 << i) - 1 for i in range(7)])
    assert np.array_equal(got1, got2)


def test_dense_cache_is_one_page_a_stream():
    """The dense verify attention and the paged call on the same memory: page_size = L_cap, page s for stream s."""
    import paper_2510_25739_b200 as hawk
    S, K, H, D, cap = 6, 5, 4, 64, 208
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn((S, K, H, D), device="cuda", generator=g).bfloat16()
    kc, vc = (torch.randn((S, H, cap, D), device="cuda", generator=g).bfloat16() for _ in range(2))
    pre = torch.tensor([0, 5, 100, 203, 31, 64], dtype=torch.int32, device="cuda")
    dense = hawk.verify_attn(q, kc, vc, pre, 203, D ** -0.5)
    out = hawk.paged_attn(q.reshape(S * K, H, D), kc, vc, torch.arange(S, dtype=torch.int32, device="cuda")[:, None],
                          torch.arange(0, S * K + 1, K, dtype=torch.int32, device="cuda"), pre + K, K, cap, D ** -0.5)
    a, b = f64(dense).reshape(-1), f64(out).reshape(-1)
    # the same products in the same order within a tile; items may be cut at other tiles
    assert np.linalg.norm(a - b) <= 2 * half_step(torch.bfloat16) * np.linalg.norm(a)


def test_loose_bounds_change_nothing_but_the_launch():
    """max_new and max_kv are upper bounds."""
    b = Batch([1, 5], [40, 333], 4, 4, 64, 16, seed=16)
    b.block_table = torch.nn.functional.pad(b.block_table, (0, 40), value=-1)
    _check(b, max_new=8, max_kv=900)


def test_shared_prefix_pages():
    """Two streams whose tables name the same pages."""
    b = Batch([2, 2], [96, 96], 2, 2, 64, 16, seed=17)
    b.block_table[1] = b.block_table[0]
    _check(b)


@pytest.mark.parametrize("n", [4, 100])
def test_pages_far_into_a_large_cache(n):
    """Element offsets past 2^31 (a cache of 4.5 GB a tensor); a head whose keys are past it too."""
    D, page, H_kv = 128, 16, 2
    pages = (1 << 31) // (H_kv * page * D) + 40
    b = Batch([n, 1], [n + 60, 35], 2, H_kv, D, page, seed=18)
    d = b.cuda()
    far = torch.arange(pages - b.n_pages, pages, dtype=torch.int32)
    table = b.block_table.clone()
    table[table >= 0] = far[table[table >= 0].long()]
    for name in ("k_pages", "v_pages"):
        big = torch.empty((pages, H_kv, page, D), dtype=b.dt, device="cuda")
        big[pages - b.n_pages:] = getattr(d, name)
        setattr(d, name, big)
    d.block_table = table.cuda()
    got, status = _run(b, dev=d)
    assert status == 0
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), D ** -0.5)
    _compare(got, want, size, b.dt)


def test_what_the_device_finds_wrong_is_flagged():
    import paper_2510_25739_b200.binding as hb
    b = Batch([2, 90, 3], [40, 95, 20], 2, 2, 64, 16, seed=19)
    want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  b.kv_len.numpy(), 64 ** -0.5)
    # a page id out of range: that stream's rows are not valid, the others' are
    for s in (0, 1):
        d = b.cuda()
        d.block_table[s, 1] = b.n_pages + 5
        got, status = _run(b, dev=d)
        assert status == hb.DEV_BAD_PAGE
        ok = np.ones(b.T, dtype=bool)
        ok[int(b.row_begin[s]):int(b.row_begin[s + 1])] = False
        h = half_step(b.dt)
        assert (np.abs(got - want)[ok] <= (h * np.abs(want) + (h + 2.0 ** -11) * size)[ok]).all()
    # more keys than the bound, a negative count: clamped
    for bad in (1000, -3):
        d = b.cuda()
        d.kv_len[2] = bad
        _, status = _run(b, dev=d, max_kv=95)
        assert status & hb.DEV_BAD_PREFIX
    # rows that run backwards or past the call's, a stream longer than the bound: that stream is skipped
    d = b.cuda()
    d.row_begin[1] = 200
    got, status = _run(b, dev=d)
    assert status == hb.DEV_BAD_ROWS and (got[:92] == 7.0).all()
    d = b.cuda()
    got, status = _run(b, dev=d, max_new=50)
    assert status == hb.DEV_BAD_ROWS and (got[2:92] == 7.0).all() and (got[92:] != 7.0).any()


def test_captured_and_replayed():
    """A captured call on another stream; replays see new queries and new lengths."""
    import paper_2510_25739_b200 as hawk
    b = Batch([3, 120, 1], [200, 150, 64], 4, 2, 64, 16, seed=20)
    d = b.cuda()
    out = torch.zeros((b.T, b.H * b.D), dtype=b.dt, device="cuda")
    ws = torch.empty(max(16, hawk.paged_attn_workspace_bytes(b.S, b.T, 120, 4, 2, 64, 200)), dtype=torch.uint8, device="cuda")

    def call():
        hawk.paged_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, 120, 200, b.D ** -0.5, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    b2 = Batch([3, 120, 1], [200, 150, 64], 4, 2, 64, 16, seed=21)
    d.q.copy_(b2.q)
    d.kv_len.copy_(torch.tensor([180, 140, 3], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    want, size = paged.paged_attn(f64(b2.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), b.row_begin.numpy(),
                                  np.array([180, 140, 3]), b.D ** -0.5)
    _compare(f64(out).reshape(b.T, b.H, b.D), want, size, b.dt)


def test_two_calls_at_once():
    """Two streams of the GPU, a workspace each: the same results as one after the other."""
    import paper_2510_25739_b200 as hawk
    bs = [Batch([5] * 30, [500] * 30, 4, 4, 64, 16, seed=22 + i) for i in range(2)]
    ds = [b.cuda() for b in bs]
    alone = [_run(b, dev=d)[0] for b, d in zip(bs, ds)]
    streams = [torch.cuda.Stream() for _ in bs]
    outs = [torch.zeros((b.T, b.H * b.D), dtype=b.dt, device="cuda") for b in bs]
    torch.cuda.synchronize()
    for _ in range(10):
        for b, d, o, st in zip(bs, ds, outs, streams):
            with torch.cuda.stream(st):
                hawk.paged_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, 5, 500, b.D ** -0.5, out=o)
    torch.cuda.synchronize()
    for b, a, o in zip(bs, alone, outs):
        assert np.array_equal(a, f64(o).reshape(b.T, b.H, b.D))
