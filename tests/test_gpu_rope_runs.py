"""hawk_qk_norm_rope and hawk_rope_append on prompts: calls of so many rows that a block takes a run of them, with the table lines of
its run in shared memory.  Both calls take the variant from 296 * par rows on, par being the rows that a block has in hand at
once (256 lanes over the lanes of a row's heads, in as few rounds as a block needs or up to three more).  Runs of an odd and an even number of
passes, short last blocks, several rounds of heads, heads that leave lanes idle.  Bounds as in test_gpu_rope_append.py."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_25739_b200 import binding
from tests._paged import DTYPES, Batch, f64, rope_table
from tests.test_gpu_rope_append import _near, _weights

pytestmark = pytest.mark.gpu


def _passes(T, heads, D):
    """Passes of a block over its run by the rule of the launch (1: the variant for few rows)."""
    lh = D // 16
    fit = 256 // lh
    least = -(-heads // fit)
    best, par = 0, 0
    for rounds in range(least, min(least + 3, heads) + 1):
        lanes = -(-heads // rounds) * lh
        p = min(256 // lanes, 64)
        used = 1000 * p * heads * lh // (256 * rounds)
        if rounds == least or (used > best + best // 10 and T >= 296):
            best, par = used, p
    return min(-(-T // (296 * par)), max(32 // par, 1)), par


def _setup(g, T, H, H_kv, D, rot, norm, dt, per_head):
    w = [_weights(g, h, D, per_head, dt, m) for m in (1.0, 0.0) for h in (H, H_kv)] if norm != "none" else [None] * 4
    if norm == "rms":
        w[2] = w[3] = None
    position = torch.randint(0, 40, (T,), generator=g, dtype=torch.int32)
    return w, position, rope_table(40, rot) if rot else None


@pytest.mark.parametrize("T,H,H_kv,D,rot,interleaved,passes", [
    (700, 32, 32, 128, 64, False, 3),    # two rounds of heads, a row in hand; the last block has one row
    (500, 32, 32, 128, 128, True, 2),
    (1000, 24, 24, 128, 32, False, 2),   # 48 heads: three rounds of 16 and two rows in hand
    (901, 40, 20, 64, 32, True, 4),
    (1300, 20, 20, 64, 0, False, 2),     # three rows in hand, two rounds
    (1400, 32, 32, 128, 16, False, 5),
    (5000, 2, 2, 64, 16, False, 2),      # 16 rows in hand
    (6001, 4, 2, 64, 16, True, 3),       # ten rows in hand and 16 lanes without a row
    (2500, 5, 0, 128, 16, False, 2),     # queries alone
    (12000, 32, 32, 64, 0, False, 32),   # more than one wave: the longest run
])
@pytest.mark.parametrize("norm,dtype,per_head", [("none", "bf16", False), ("rms", "fp16", True), ("layer", "bf16", True),
                                                 ("rms", "bf16", False), ("layer", "fp16", False)])
def test_norm_rope(T, H, H_kv, D, rot, interleaved, passes, norm, dtype, per_head):
    import paper_2510_25739_b200 as hawk
    assert _passes(T, H + H_kv, D)[0] == passes
    g = torch.Generator().manual_seed(T)
    dt = DTYPES[dtype]
    packed = (3 * torch.randn((T, H + H_kv + 1, D), generator=g) + 0.5).to(dt)
    q, k = packed[:, :H], packed[:, H:H + H_kv] if H_kv else None
    w, position, table = _setup(g, T, H, H_kv, D, rot, norm, dt, per_head)
    dev = packed.cuda()
    c = [None if x is None else x.cuda() for x in w]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(norm=norm, eps=1e-5, q_weight=c[0], k_weight=c[1] if H_kv else None, q_bias=c[2], k_bias=c[3] if H_kv else None,
                interleaved=interleaved, dev_status=status)
    qc, kc = dev[:, :H], dev[:, H:H + H_kv] if H_kv else None
    where = (position.cuda(), table.cuda()) if rot else (None, None)
    qo, ko = hawk.qk_norm_rope(qc, kc, *where, **args)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for x, o, wt, bias in ((q, qo, w[0], w[2]), (k, ko, w[1], w[3])):
        if x is None:
            assert o is None
            continue
        want, size = paged.norm_rope(f64(x), position.numpy(), None if table is None else table.numpy(), norm, 1e-5,
                                     None if wt is None else f64(wt), None if bias is None else f64(bias), interleaved)
        _near(f64(o), want, size, dt, D)
    # in place: the same bits, and what lies behind the two tensors untouched
    hawk.qk_norm_rope(qc, kc, *where, q_out=qc, k_out=kc, **args)
    assert torch.equal(qc, qo) and (kc is None or torch.equal(kc, ko)) and torch.equal(dev[:, H + H_kv:].cpu(), packed[:, H + H_kv:])


def test_positions_out_of_range():
    """Clamped and flagged, in whichever row of a run."""
    import paper_2510_25739_b200 as hawk
    g = torch.Generator().manual_seed(4)
    q = torch.randn((700, 64, 128), generator=g).bfloat16().cuda()
    table = rope_table(40, 64).cuda()
    good = torch.randint(0, 40, (700,), generator=g, dtype=torch.int32)
    for row, bad, clamped in ((0, -5, 0), (338, 40, 39), (699, 2 ** 31 - 1, 39)):
        position, near = good.clone(), good.clone()
        position[row], near[row] = bad, clamped
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        a, _ = hawk.qk_norm_rope(q, None, position.cuda(), table, dev_status=status)
        assert int(status.item()) == binding.DEV_BAD_POSITION
        b, _ = hawk.qk_norm_rope(q, None, near.cuda(), table)
        assert torch.equal(a, b)


@pytest.mark.parametrize("new,kv,H,H_kv,D,page,rot,interleaved,layout,passes", [
    ([300, 0, 257, 1, 190], [300, 9, 600, 77, 700], 32, 8, 128, 24, 64, False, "hrd", 2),
    ([513, 90], [513, 400], 20, 20, 64, 16, 32, True, "kv", 3),
    ([1500, 0, 1, 1700, 2600], [1600, 3, 1, 1700, 3000], 2, 1, 64, 64, 16, False, "rhd", 2),
    ([700] * 9 + [41], [800] * 9 + [50], 0, 2, 64, 16, 16, True, "hrd", 2),
    ([30] * 31, [200] * 31, 32, 16, 128, 8, 0, False, "hrd", 4),
])
@pytest.mark.parametrize("norm,dtype", [("none", "fp16"), ("rms", "bf16"), ("layer", "fp16")])
def test_append(new, kv, H, H_kv, D, page, rot, interleaved, layout, passes, norm, dtype):
    """Prompts into the cache: runs that cross streams and pages, rows of nobody in front and behind; everything else keeps its bits."""
    import paper_2510_25739_b200 as hawk
    b = Batch(new, kv, max(H, 1), H_kv, D, page, dtype, seed=34, layout=layout, front=2, back=3, packed=True, poison=5.0)
    assert _passes(b.T, H + 2 * H_kv, D)[0] == passes
    g = torch.Generator().manual_seed(5)
    w, position, table = _setup(g, b.T, max(H, 1), H_kv, D, rot, norm, b.dt, True)
    d = b.cuda()
    c = [None if x is None else x.cuda() for x in w]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full((b.T, H, D), 9.0, dtype=b.dt, device="cuda") if H else None
    where = (position.cuda(), table.cuda()) if rot else (None, None)
    r = hawk.rope_append(d.q if H else None, d.k, d.v, *where, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len, norm=norm,
                         eps=1e-5, q_weight=c[0] if H else None, k_weight=c[1], q_bias=c[2] if H else None, k_bias=c[3],
                         interleaved=interleaved, q_out=q_out, dev_status=status)
    torch.cuda.synchronize()
    assert r is q_out and int(status.item()) == 0
    n = [None if x is None else f64(x) for x in w]
    tab = None if table is None else table.numpy()
    places = np.array(paged.cache_rows(b.row_begin, b.kv_len))
    t, s, row = places.T
    if H:
        q, qs = paged.norm_rope(f64(b.q), position.numpy(), tab, norm, 1e-5, n[0], n[2], interleaved)
        got = f64(q_out)
        _near(got[t], q[t], qs[t], b.dt, D)
        assert (np.delete(got, t, 0) == 9.0).all()
    k, ks = paged.norm_rope(f64(b.k), position.numpy(), tab, norm, 1e-5, n[1], n[3], interleaved)
    pg, off = b.block_table.numpy()[s, row // page], row % page
    got_k, got_v = d.k_pages.cpu().clone(), d.v_pages.cpu().clone()
    _near(f64(got_k)[pg, :, off], k[t], ks[t], b.dt, D)
    assert torch.equal(got_v[pg, :, off], b.v[t])
    got_k[pg, :, off], got_v[pg, :, off] = b.k_pages[pg, :, off], b.v_pages[pg, :, off]
    assert torch.equal(got_k, b.k_pages) and torch.equal(got_v, b.v_pages)
