"""GPU parity of hawk_paged_attn over its kernels and launch shapes, against the plain 64-bit form: every row count of the
narrow tcgen05 kernel, items cut between blocks, scores that keep moving the softmax's shift, batches of hundreds of streams,
wide query groups, trees of many rows.  Bounds as in test_gpu_paged_attn.py (derived there); where a test makes its own scores it
keeps sum |q k| scale below the 32 that those bounds count on, and checks that it does."""
import numpy as np
import pytest
import torch

from tests._paged import Batch, f64
from tests.test_gpu_paged_attn import _binary_tree, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group", [(1, 1), (1, 7), (9, 1), (16, 1), (17, 1), (4, 5), (32, 1), (33, 1), (8, 8), (64, 1), (3, 20)])
def test_few_long_streams(n, group, D, dtype):
    """Few items over many keys: the narrow tcgen05 kernel at 16, 32 and 64 rows, each item cut into several shares."""
    _check(Batch([n] * 3, [3000, max(n, 131), 1777], 2 * group, 2, D, 16, dtype, seed=40))


@pytest.mark.parametrize("n,kv", [(30, 500), (40, 700), (64, 301)])
def test_many_items_of_many_rows(n, kv):
    """More items than blocks, so that a block walks through several and shares begin inside them; every stream another length."""
    rng = np.random.default_rng(n)
    S = 12
    _check(Batch([int(x) for x in rng.integers(1, n + 1, S - 1)] + [n], [int(x) for x in rng.integers(n, kv + 1, S)], 20, 20, 128, 16,
                 seed=41))


@pytest.mark.parametrize("n,D", [(7, 64), (7, 128), (12, 64), (12, 128), (20, 64), (24, 128), (30, 64), (40, 64), (60, 64)])
def test_many_short_items(n, D):
    """Thousands of items of one or two 128-key tiles: equal shares of warps, one to four column tiles an item, or two items."""
    rng = np.random.default_rng(n)
    S = 64
    _check(Batch([int(x) for x in rng.integers(0, n + 1, S - 1)] + [n], [int(x) for x in rng.integers(n, 200, S - 1)] + [200], 20, 20, D,
                 8, seed=53))


@pytest.mark.parametrize("D", [64, 128])
def test_last_tiles_of_every_fill(D):
    """Keys that end at, before and behind the boundaries of a 128-key tile, of a page and of a box."""
    kv = [1100, 128, 127, 129, 1, 136, 135, 137, 256, 255, 257, 1025]
    _check(Batch([min(30, x) for x in kv], kv, 2, 2, D, 24, seed=42))


@pytest.mark.parametrize("n", [12, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_long_streams_with_rows_that_see_nothing(n, D):
    """Streams with fewer keys than rows, with no keys and without rows between long ones."""
    b = Batch([n, n, 0, n, n], [2500, n - 5, 3, 0, 2], 2, 2, D, 16, seed=43, front=2, back=2)
    _check(b)
    got, _ = _run(b)
    for s in (1, 3, 4):
        r0 = int(b.row_begin[s])
        assert (got[r0:r0 + n - b.kv[s]] == 0).all()


@pytest.mark.parametrize("n,H,H_kv,D", [(22, 2, 2, 128), (40, 1, 1, 64), (64, 1, 1, 128), (20, 6, 2, 64)])
def test_trees_over_long_prefixes(n, H, H_kv, D):
    _check(Batch([n, n // 2], [n + 2000, n // 2 + 1500], H, H_kv, D, 16, seed=44), _binary_tree(n))


@pytest.mark.parametrize("n,H,H_kv,D", [(64, 8, 2, 64), (40, 16, 1, 128), (63, 4, 2, 128), (30, 24, 2, 64)])
def test_trees_of_many_rows(n, H, H_kv, D):
    """More than 64 rows per kv head under a mask: the wide kernel reads it too."""
    masks = _binary_tree(n)
    masks[n // 2] = 0  # a node that sees the prefix alone
    _check(Batch([n, n, 1], [n + 500, n, 1], H, H_kv, D, 16, seed=45), masks)


@pytest.mark.parametrize("n,H,H_kv", [(1, 100, 1), (2, 200, 2), (5, 128, 1), (1, 65, 1)])
def test_wide_groups(n, H, H_kv):
    """More query heads per kv head than the few-row kernels take: every stream is the wide kernel's."""
    _check(Batch([n, 1, 0], [n + 777, 40, 2], H, H_kv, 64, 16, seed=46))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [3, 16, 31, 50, 150])
def test_scores_that_keep_rising(n, D):
    """The best score so far grows by 24 over the keys (35 in log2 units): the shift moves again and again, and with it every sum
    and accumulator; in one stream the scores fall instead."""
    b = Batch([n, n], [2200, 1500], 2, 2, D, 16, seed=47)
    g = torch.Generator().manual_seed(48)
    base = torch.randint(0, 2, (D,), generator=g).float() * 2 - 1
    b.q = (base + 0.1 * torch.randn(b.q.shape, generator=g)).to(b.dt)
    for s, kv in enumerate(b.kv):
        for j in range(kv):
            ramp = 24 * D ** -0.5 * (j / kv if s == 0 else 1 - j / kv)
            k = base * ramp + 0.1 * torch.randn((b.H_kv, D), generator=g)
            b.k_pages[int(b.block_table[s, j // b.page]), :, j % b.page] = k.to(b.dt)
    reach = np.nanmax(np.abs(f64(b.k_pages)), axis=(0, 1, 2)) @ np.abs(f64(b.q)).max(axis=(0, 1)) * D ** -0.5
    assert np.isfinite(reach)
    per_key = np.abs(f64(b.q)).reshape(-1, D) @ np.abs(np.nan_to_num(f64(b.k_pages))).reshape(-1, D).T * D ** -0.5
    assert per_key.max() < 32
    _check(b)


@pytest.mark.parametrize("S,n", [(400, 1), (1000, 2), (4096, 1)])
def test_hundreds_of_streams(S, n):
    """More streams than threads of a block: the prefix sum takes several rounds.  Some are idle."""
    rng = np.random.default_rng(S)
    new = [int(x) for x in rng.integers(0, n + 1, S)]
    new[-1] = n
    _check(Batch(new, [int(x) for x in rng.integers(n, 60, S)], 2, 1, 64, 8, seed=49))


def test_hundreds_of_streams_with_chunks():
    """The list of the wide kernel's blocks over several hundred streams, more of them than one wave of blocks holds."""
    rng = np.random.default_rng(50)
    new = [int(x) for x in rng.choice([0, 1, 5, 70, 130], 500)]
    _check(Batch(new, [n + int(x) for n, x in zip(new, rng.integers(0, 90, 500))], 2, 2, 64, 16, seed=50))


def test_long_streams_with_chunks_between():
    """Both tcgen05 kernels in one call."""
    _check(Batch([20, 150, 1, 64, 300], [2500, 900, 2000, 64, 400], 2, 2, 128, 16, seed=51, front=1, back=1, packed=True))


def test_replays_with_other_lengths():
    """Shares are cut on the device: a captured call follows lengths and row counts that change under it, idle streams too."""
    import paper_2510_25739_b200 as hawk
    from oracle import paged
    H, D = 2, 128
    b = Batch([40, 40], [2600, 2600], H, H, D, 16, seed=52)
    d = b.cuda()
    out = torch.zeros((b.T, H * D), dtype=b.dt, device="cuda")
    ws = torch.empty(hawk.paged_attn_workspace_bytes(2, b.T, 40, H, H, D, 2600), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()

    def call():
        hawk.paged_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, 40, 2600, D ** -0.5, out=out, workspace=ws)

    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    h = 2.0 ** -8
    for begin, kv in (([0, 40, 80], [2600, 1300]), ([0, 0, 33], [2600, 2599]), ([5, 6, 6], [131, 9]), ([0, 17, 57], [17, 200]),
                      ([0, 0, 0], [1, 1])):
        d.row_begin.copy_(torch.tensor(begin, dtype=torch.int32))
        d.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        want, size = paged.paged_attn(f64(b.q), f64(b.k_pages), f64(b.v_pages), b.block_table.numpy(), np.array(begin), np.array(kv),
                                      D ** -0.5)
        got, rows = f64(out).reshape(b.T, H, D), slice(begin[0], begin[2])
        assert (np.delete(got, np.arange(begin[0], begin[2]), 0) == 7).all()
        assert (np.abs(got - want)[rows] <= (h * np.abs(want) + (h + 2.0 ** -11) * size)[rows]).all()
