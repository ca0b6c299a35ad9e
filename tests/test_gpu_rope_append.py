"""GPU parity of hawk_qk_norm_rope and hawk_rope_append against the plain 64-bit form, and the calls around the paged cache
used together.

Bounds.  One rounding to the 16-bit type (half step h of the value; below the type's normal range half of its smallest
step), and fp32 arithmetic before it: at most D + 16 roundings of terms no larger than `size` (the norm's sum of D squares
counts half, under the root), so |got - want| <= h |want| + (D + 16) 2^-24 size + tiny.
"""
import numpy as np
import pytest
import torch

from oracle import paged
from tests._paged import DTYPES, Batch, f64, half_step, rope_table

pytestmark = pytest.mark.gpu


def _near(got, want, size, dt, D):
    bound = half_step(dt) * np.abs(want) + (D + 16) * 2.0 ** -24 * size + torch.finfo(dt).smallest_normal * half_step(dt)
    err = np.abs(got - want)
    assert (err <= bound).all(), (err.max(), np.unravel_index(np.argmax(err - bound), err.shape))


def _weights(g, heads, D, per_head, dt, mean):
    return (mean + 0.2 * torch.randn((heads, D) if per_head else (D,), generator=g)).to(dt)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (64, 64, True), (128, 128, False), (128, 128, True), (128, 64, False),
                                               (128, 16, True), (64, 32, True), (64, 48, False), (64, 0, False)])
def test_norm_rope(dtype, norm, D, rot, interleaved):
    import paper_2510_25739_b200 as hawk
    g = torch.Generator().manual_seed(D + rot)
    dt, T, H, H_kv, per_head = DTYPES[dtype], 13, 5, 3, rot % 64 == 0
    packed = (3 * torch.randn((T, H + H_kv + 1, D), generator=g) + 0.5).to(dt)
    q, k = packed[:, :H], packed[:, H:H + H_kv]
    position = torch.randint(0, 50, (T,), generator=g, dtype=torch.int32)
    table = rope_table(50, rot, grid=8 if rot == 64 else 0) if rot else None
    w = [_weights(g, h, D, per_head, dt, m) for m in (1.0, 0.0) for h in (H, H_kv)] if norm != "none" else [None] * 4
    if norm == "rms":
        w[2] = w[3] = None
    elif norm == "layer" and D == 64:
        w[3] = None  # a bias for the queries only
    dev = packed.cuda()
    qc, kc = dev[:, :H], dev[:, H:H + H_kv]
    c = [None if x is None else x.cuda() for x in w]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(norm=norm, eps=1e-5, q_weight=c[0], k_weight=c[1], q_bias=c[2], k_bias=c[3], interleaved=interleaved)
    qo, ko = hawk.qk_norm_rope(qc, kc, position.cuda() if rot else None, None if table is None else table.cuda(),
                               dev_status=status, **args)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for x, o, wt, bias in ((q, qo, w[0], w[2]), (k, ko, w[1], w[3])):
        want, size = paged.norm_rope(f64(x), position.numpy(), None if table is None else table.numpy(), norm, 1e-5,
                                     None if wt is None else f64(wt), None if bias is None else f64(bias), interleaved)
        _near(f64(o), want, size, dt, D)
    # in place: the same bits, and what lies between the two tensors untouched
    hawk.qk_norm_rope(qc, kc, position.cuda() if rot else None, None if table is None else table.cuda(), q_out=qc, k_out=kc, **args)
    assert torch.equal(qc, qo) and torch.equal(kc, ko) and torch.equal(dev[:, H + H_kv:].cpu(), packed[:, H + H_kv:])


@pytest.mark.parametrize("T,H,H_kv,D", [(1, 1, 1, 64), (1, 32, 32, 128), (257, 1, 1, 64), (40, 40, 8, 128), (5, 70, 70, 64), (3, 7, 0, 64),
                                        (3, 0, 7, 128)])
def test_norm_rope_sizes(T, H, H_kv, D):
    """One row to many, one head to more than a block holds at once, one of the two tensors alone."""
    import paper_2510_25739_b200 as hawk
    g = torch.Generator().manual_seed(T)
    q, k = (torch.randn((T, h, D), generator=g).bfloat16() if h else None for h in (H, H_kv))
    position = torch.arange(T, dtype=torch.int32) % 31
    table = rope_table(31, D)
    w = torch.ones(D).bfloat16()
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    qo, ko = hawk.qk_norm_rope(up(q), up(k), position.cuda(), table.cuda(), norm="rms", q_weight=w.cuda(), k_weight=w.cuda())
    for x, o in ((q, qo), (k, ko)):
        if x is None:
            assert o is None
            continue
        want, size = paged.norm_rope(f64(x), position.numpy(), table.numpy(), "rms", 1e-6, f64(w))
        _near(f64(o), want, size, torch.bfloat16, D)


def test_position_out_of_range_is_clamped_and_flagged():
    import paper_2510_25739_b200 as hawk
    import paper_2510_25739_b200.binding as hb
    q = torch.randn((3, 2, 64)).bfloat16().cuda()
    table = rope_table(10, 64).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    a, _ = hawk.qk_norm_rope(q, None, torch.tensor([-4, 3, 99], dtype=torch.int32).cuda(), table, dev_status=status)
    assert int(status.item()) == hb.DEV_BAD_POSITION
    b, _ = hawk.qk_norm_rope(q, None, torch.tensor([0, 3, 9], dtype=torch.int32).cuda(), table)
    assert torch.equal(a, b)


def _append_want(b, position, table, norm, eps, wq, wk, bq, bk, interleaved):
    q, qs = paged.norm_rope(f64(b.q), position, table, norm, eps, wq, bq, interleaved)
    k, ks = paged.norm_rope(f64(b.k), position, table, norm, eps, wk, bk, interleaved)
    return q, qs, k, ks


@pytest.mark.parametrize("dtype,layout,D,H,H_kv,page", [("bf16", "hrd", 64, 4, 4, 16), ("fp16", "rhd", 128, 8, 2, 24), ("bf16", "kv", 64, 5, 1, 7),
                                                        ("fp16", "hrd", 64, 20, 20, 1), ("bf16", "rhd", 128, 40, 40, 64)])
@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
def test_append(dtype, layout, D, H, H_kv, page, norm):
    """Ragged rows, an idle stream, rows of nobody, pages of odd sizes: the new rows land, everything else keeps its bits."""
    import paper_2510_25739_b200 as hawk
    new, kv = [3, 0, 1, 9, 17], [40, 5, 1, 9, 100]
    b = Batch(new, kv, H, H_kv, D, page, dtype, seed=30, layout=layout, front=2, back=3, packed=True, poison=5.0)
    g = torch.Generator().manual_seed(3)
    w = [_weights(g, h, D, True, b.dt, m) for m in (1.0, 0.0) for h in (H, H_kv)] if norm != "none" else [None] * 4
    if norm == "rms":
        w[2] = w[3] = None
    position = torch.randint(0, 60, (b.T,), generator=g, dtype=torch.int32)
    table = rope_table(60, D, grid=8)
    d = b.cuda()
    q_out = torch.full((b.T, H, D), 9.0, dtype=b.dt, device="cuda")
    c = [None if x is None else x.cuda() for x in w]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = hawk.rope_append(d.q, d.k, d.v, position.cuda(), table.cuda(), d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len,
                         norm=norm, eps=1e-5, q_weight=c[0], k_weight=c[1], q_bias=c[2], k_bias=c[3], q_out=q_out, dev_status=status)
    torch.cuda.synchronize()
    assert r is q_out and int(status.item()) == 0
    q, qs, k, ks = _append_want(b, position.numpy(), table.numpy(), norm, 1e-5, *[None if x is None else f64(x) for x in w], False)
    got_q, got_k, got_v = f64(q_out), d.k_pages.cpu().clone(), d.v_pages.cpu().clone()
    owned = [t for t, _, _ in paged.cache_rows(b.row_begin, b.kv_len)]
    _near(got_q[owned], q[owned], qs[owned], b.dt, D)
    assert (np.delete(got_q, owned, 0) == 9.0).all()
    for t, s, row in paged.cache_rows(b.row_begin, b.kv_len):
        pg, off = int(b.block_table[s, row // page]), row % page
        _near(f64(got_k[pg, :, off]), k[t], ks[t], b.dt, D)
        assert torch.equal(got_v[pg, :, off], b.v[t])
        got_k[pg, :, off] = b.k_pages[pg, :, off]
        got_v[pg, :, off] = b.v_pages[pg, :, off]
    assert torch.equal(got_k, b.k_pages) and torch.equal(got_v, b.v_pages)


def test_append_many_streams_and_no_queries():
    """More streams than a block has threads, most of them idle or with one row; keys and values only."""
    import paper_2510_25739_b200 as hawk
    rng = np.random.default_rng(1)
    new = [int(x) for x in rng.integers(0, 3, 700)]
    kv = [n + int(x) for n, x in zip(new, rng.integers(0, 5, 700))]
    b = Batch(new, kv, 2, 2, 64, 4, seed=31, poison=5.0)
    d = b.cuda()
    assert hawk.rope_append(None, d.k, d.v, None, None, d.k_pages, d.v_pages, d.block_table, d.row_begin, d.kv_len) is None
    got_k, got_v = d.k_pages.cpu(), d.v_pages.cpu()
    for t, s, row in paged.cache_rows(b.row_begin, b.kv_len):
        b.k_pages[int(b.block_table[s, row // 4]), :, row % 4] = b.k[t]
        b.v_pages[int(b.block_table[s, row // 4]), :, row % 4] = b.v[t]
    assert torch.equal(got_k, b.k_pages) and torch.equal(got_v, b.v_pages)


def test_append_skips_and_flags_what_has_no_place():
    import paper_2510_25739_b200 as hawk
    import paper_2510_25739_b200.binding as hb
    b = Batch([2, 2, 2], [20, 20, 20], 2, 2, 64, 16, seed=32, poison=5.0)
    d = b.cuda()
    before = d.k_pages.clone(), d.v_pages.clone()
    for bits, table, lens in ((hb.DEV_BAD_PAGE, b.n_pages, 20), (hb.DEV_BAD_PAGE, -1, 20), (hb.DEV_BAD_PREFIX, 0, 10 ** 6), (hb.DEV_BAD_PREFIX, 0, -1)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        tb, ln = d.block_table.clone(), d.kv_len.clone()
        tb[:] = table
        ln[:] = lens
        q = hawk.rope_append(d.q, d.k, d.v, None, None, d.k_pages, d.v_pages, tb, d.row_begin, ln, dev_status=status)
        assert int(status.item()) == bits
        assert torch.equal(q, d.q)  # without norm and rotation the queries come back as they were
        assert torch.equal(d.k_pages, before[0]) and torch.equal(d.v_pages, before[1])


def test_append_into_the_dense_cache_of_the_verify_attention():
    """A dense cache [S][H_kv][L_cap][D] is one page a stream: rope_append writes the block's rows, verify_attn reads them."""
    import paper_2510_25739_b200 as hawk
    S, K, H, D, cap = 4, 5, 3, 64, 100  # (a page of 100 rows: the append takes any size)
    b = Batch([K] * S, [K, 30, 100, 64], H, H, D, cap, seed=33)
    d = b.cuda()
    kc, vc = torch.randn((S, H, cap, D), device="cuda").bfloat16(), torch.randn((S, H, cap, D), device="cuda").bfloat16()
    table = rope_table(120, D)
    position = torch.cat([torch.arange(l - K, l) for l in b.kv]).int()
    ident = torch.arange(S, dtype=torch.int32, device="cuda")[:, None]
    q = hawk.rope_append(d.q, d.k, d.v, position.cuda(), table.cuda(), kc, vc, ident, d.row_begin, d.kv_len)
    out = hawk.verify_attn(q.reshape(S, K, H, D), kc, vc, d.kv_len - K, cap - K, D ** -0.5)
    torch.cuda.synchronize()
    want, size = paged.paged_attn(f64(q), f64(kc), f64(vc), ident.cpu().numpy(), b.row_begin.numpy(), b.kv_len.numpy(), D ** -0.5)
    got = f64(out).reshape(S * K, H, D)
    h = half_step(torch.bfloat16)
    assert (np.abs(got - want) <= h * np.abs(want) + (h + 2.0 ** -11) * size).all()
    k, ks = paged.norm_rope(f64(b.k), position.numpy(), table.numpy())
    for t, s, row in paged.cache_rows(b.row_begin, b.kv_len):
        _near(f64(kc[s, :, row]), k[t], ks[t], torch.bfloat16, D)


def test_generation_over_the_paged_cache():
    """Used together: a prompt enters in two chunks of unequal streams, a drafted block is verified, its accepted part is
    kept and single tokens follow; every step's attention against the plain form over the whole history."""
    import paper_2510_25739_b200 as hawk
    S, H, H_kv, D, page, dt = 3, 4, 2, 64, 16, torch.bfloat16
    g = torch.Generator().manual_seed(77)
    table = rope_table(300, D, grid=16)
    w = (1 + 0.2 * torch.randn((D,), generator=g)).to(dt)
    width = 20
    pages = S * width
    kp, vp = (torch.full((pages, H_kv, page, D), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    tables = torch.randperm(pages, generator=g).int().reshape(S, width)
    lens = [0] * S
    for step, new in enumerate([[70, 3, 120], [5, 90, 64], [5, 5, 5], [1, 1, 0], [1, 1, 1]]):
        if step == 3:
            lens = [l - 2 for l in lens]  # two drafts of each block were rejected: their rows are written over
        lens = [l + n for l, n in zip(lens, new)]
        T = sum(new)
        qkv = torch.randn((T, H + 2 * H_kv, D), generator=g).to(dt).cuda()
        begin = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        position = torch.cat([torch.arange(l - n, l) for l, n in zip(lens, new)]).int()
        kv = torch.tensor(lens, dtype=torch.int32)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        q = hawk.rope_append(qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:], position.cuda(), table.cuda(), kp, vp, tables.cuda(),
                             begin.cuda(), kv.cuda(), norm="rms", q_weight=w.cuda(), k_weight=w.cuda(), dev_status=status)
        out = hawk.paged_attn(q, kp, vp, tables.cuda(), begin.cuda(), kv.cuda(), max(new), max(lens), D ** -0.5, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        want, size = paged.paged_attn(f64(q), f64(kp), f64(vp), tables.numpy(), begin.numpy(), kv.numpy(), D ** -0.5)
        got = f64(out).reshape(T, H, D)
        h = half_step(dt)
        assert (np.abs(got - want) <= h * np.abs(want) + (h + 2.0 ** -11) * size).all()
        assert np.linalg.norm(got - want) <= (2 * h + 2.0 ** -11) * np.linalg.norm(want)
