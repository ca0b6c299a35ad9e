"""Measured cases of the operators around the paged key/value cache.

Three operators, one `run` each:
  norm_rope  qk_norm_rope: norm of every query and key head, then the position rotation, dense in and out
  append     rope_append: the same on the way of new keys and values into a paged cache
  attn       paged_attn: attention of a chunk of new tokens (or of a candidate tree) over the paged cache

The batches are ragged where a case says so: stream s brings new_s rows, `row_begin` holds their running sum, `kv_len` the
stream's keys including the new ones, and a few rows behind the last stream belong to nobody (a padded batch).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
SPARE_ROWS = 3  # rows behind the last stream of a ragged batch
EPS = 1e-5


def _case(name, op, dtype, streams, new, heads, kv_heads, dim, kv, page, ragged=False, tree=False, norm="none", bias=False,
          per_head=False, interleaved=False, rot=None, grid=0, packed=False):
    return dict(name=name, op=op, dtype=dtype, streams=streams, new=new, heads=heads, kv_heads=kv_heads, dim=dim, kv=kv, page=page,
                ragged=ragged, tree=tree, norm=norm, bias=bias, per_head=per_head, interleaved=interleaved,
                rot=dim if rot is None else rot, grid=grid, packed=packed)


def listed():
    return [
        # q and k of one verify step of the XL shape: 16 guidance streams of 5 drafted rows, raster rotation of a 24-wide image
        _case("norm_rope_verify_xl", "norm_rope", "bf16", 16, 5, 20, 20, 64, 1149, 16, norm="rms", interleaved=True, grid=24,
              packed=True),
        # q and k of prompts and image prefixes entering the 7B shape: layer norm with a weight and a bias for each head
        _case("norm_rope_prefill_7b", "norm_rope", "bf16", 16, 511, 32, 32, 128, 2400, 16, ragged=True, norm="layer", bias=True,
              per_head=True, packed=True),
        # one token of one sequence (two guidance streams), the smallest call
        _case("append_decode_tiny", "append", "bf16", 2, 1, 16, 16, 64, 129, 16, interleaved=True, grid=24),
        # a full batch's verify step: 128 streams of 8 rows
        _case("append_verify_stress", "append", "bf16", 128, 8, 20, 20, 64, 1032, 32, norm="rms", interleaved=True, grid=32, packed=True),
        # prompts entering the cache in fp16 with shared key/value heads and half of each head rotated, pages of 24 rows
        _case("append_prefill_gqa", "append", "fp16", 12, 701, 32, 8, 128, 1300, 24, ragged=True, norm="rms", rot=64, packed=True),
        # one token of one sequence over a short cache, the smallest call
        _case("attn_decode_tiny", "attn", "bf16", 2, 1, 16, 16, 64, 129, 16),
        # the XL verify step: 16 streams, 5 drafted rows, 1144 cached keys
        _case("attn_verify_xl", "attn", "bf16", 16, 5, 20, 20, 64, 1149, 16),
        # the stress verify step: 128 streams, 8 drafted rows, 1024 cached keys
        _case("attn_verify_stress", "attn", "bf16", 128, 8, 20, 20, 64, 1032, 32),
        # a candidate tree of 22 nodes at the 7B shape
        _case("attn_tree_7b", "attn", "bf16", 8, 22, 32, 32, 128, 2422, 16, tree=True),
        # single tokens of few long, uneven sequences with shared key/value heads
        _case("attn_decode_long_gqa", "attn", "fp16", 7, 1, 32, 8, 128, 30011, 64, ragged=True),
        # chunks of prompts at the 7B shape over an uneven cache
        _case("attn_chunk_7b", "attn", "bf16", 5, 511, 32, 32, 128, 2911, 16, ragged=True),
        # long chunks over a long cache, shared key/value heads
        _case("attn_prefill_gqa", "attn", "bf16", 4, 2048, 32, 8, 128, 8192, 128),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("norm_rope", "append", "attn", "attn"))
    dim = rng.choice((64, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 16, 20, 32) if dim == 64 else (1, 2, 4, 8, 16, 32))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 5, 8))
    while heads > 40:
        heads -= kv_heads
    dtype = rng.choice(("bf16", "bf16", "fp16"))
    page = rng.choice((8, 16, 16, 24, 32, 64, 128, 256))
    tree = rng.random() < 0.2
    long = not tree and rng.random() < 0.4
    new = rng.randrange(7, 64) if tree else log(65, 2048) if long else log(1, 40)
    kv = new + log(1, 30000 if op == "attn" and not long else 6000)
    # what the plain form holds, at most that of the largest cases: padded scores, gathered keys, rows
    limit = max(1, min(int(4 * 32 * 2048 * 8192 / (heads * new * kv)), int(128 * 20 * 1032 * 64 * 2 / (kv_heads * kv * dim)),
                       int(16 * 511 * 64 * 128 / ((heads + 2 * kv_heads) * dim * new)), 256))
    streams = log(1, limit)
    style = dict(norm=rng.choice(("none", "rms", "layer")), interleaved=rng.random() < 0.5, per_head=rng.random() < 0.5,
                 bias=rng.random() < 0.5, rot=rng.choice((dim, dim, dim // 2, 16)), grid=rng.choice((0, 0, 24, 48)),
                 packed=rng.random() < 0.5) if op != "attn" else {}
    case = _case("", op, dtype, streams, new, heads, kv_heads, dim, kv, page, ragged=not tree and rng.random() < 0.6, tree=tree, **style)
    del case["name"]
    return case


def _lengths(case):
    """New rows and keys of every stream: the same for every seed."""
    S, new, kv = case["streams"], case["new"], case["kv"]
    if not case["ragged"]:
        return [new] * S, [kv] * S
    r = random.Random("%d %d %d" % (S, new, kv))
    ns = [r.randint(-(-new // 4), new) for _ in range(S)]
    ns[r.randrange(S)] = new
    if S >= 4:
        at = r.randrange(S)
        ns[at] = 0 if ns[at] != new else new  # a slot of the batch that is idle in this step
    ls = [r.randint(max(n, kv // 4), kv) for n in ns]
    ls[r.randrange(S)] = kv
    return ns, ls


def _parents(n):
    """A candidate tree of n nodes in breadth-first order, two children a node."""
    return [-1] + [(i - 1) // 2 for i in range(1, n)]


def _depths(n):
    return [int(math.log2(i + 1)) for i in range(n)]


def _masks(n):
    masks = []
    for i, p in enumerate(_parents(n)):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    return masks


def _table(positions, rot, grid):
    """cos | sin of every position: one axis, or (grid columns wide) half of the angles by row and half by column."""
    half = rot // 2
    at = torch.arange(positions, dtype=torch.float64, device="cuda")
    if grid:
        part = half // 2
        f = 10000.0 ** (-torch.arange(part, dtype=torch.float64, device="cuda") / part)
        angle = torch.cat([(at // grid)[:, None] * f, (at % grid)[:, None] * f], 1)
    else:
        f = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = at[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


class State:
    pass


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    st = State()
    st.case = case
    dt = DTYPES[case["dtype"]]
    S, H, Hkv, D = case["streams"], case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape, mean=0.0, std=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(mean, std, generator=g)

    ns, ls = _lengths(case)
    begin = [0]
    for n in ns:
        begin.append(begin[-1] + n)
    st.rows = begin[-1]
    T = st.rows + (SPARE_ROWS if case["ragged"] else 0)
    st.row_begin = torch.tensor(begin, dtype=torch.int32, device="cuda")
    st.kv_len = torch.tensor(ls, dtype=torch.int32, device="cuda")

    # q, k, v of the new rows: a projection's output, cut into heads (views of one buffer where the case is packed)
    if case["op"] == "attn":
        st.q = normal(T, H, D)
    elif case["packed"]:
        qkv = normal(T, H + 2 * Hkv, D)
        st.q, st.k, st.v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        st.q, st.k, st.v = normal(T, H, D), normal(T, Hkv, D), normal(T, Hkv, D)
    st.q_out = torch.zeros((T, H, D), dtype=dt, device="cuda")

    if case["op"] != "attn":
        depth = _depths(case["new"]) if case["tree"] else list(range(case["new"]))
        where = [l - n + depth[i] for n, l in zip(ns, ls) for i in range(n)] + [0] * (T - st.rows)
        st.position = torch.tensor(where, dtype=torch.int32, device="cuda")
        st.cos_sin = _table(case["kv"] + 1, case["rot"], case["grid"])
        st.q_weight = st.k_weight = st.q_bias = st.k_bias = None
        if case["norm"] != "none":
            st.q_weight = normal(*((H, D) if case["per_head"] else (D,)), mean=1.0, std=0.2)
            st.k_weight = normal(*((Hkv, D) if case["per_head"] else (D,)), mean=1.0, std=0.2)
            if case["bias"] and case["norm"] == "layer":
                st.q_bias = normal(*((H, D) if case["per_head"] else (D,)), std=0.2)
                st.k_bias = normal(*((Hkv, D) if case["per_head"] else (D,)), std=0.2)
    if case["op"] == "norm_rope":
        st.k_out = torch.zeros((T, Hkv, D), dtype=dt, device="cuda")
        return st

    # the paged cache: pages handed out in no order, the table's unused entries naming no page in particular
    page = case["page"]
    need = [-(-l // page) for l in ls]
    width = -(-case["kv"] // page)
    order = torch.randperm(sum(need) + 5, generator=g, device="cuda").int()
    table = torch.zeros((S, width), dtype=torch.int32, device="cuda")
    used = torch.arange(width, device="cuda")[None, :] < torch.tensor(need, device="cuda")[:, None]
    table[used] = order[:sum(need)]
    st.block_table = table
    st.k_pages = normal(sum(need) + 5, Hkv, page, D)
    st.v_pages = normal(sum(need) + 5, Hkv, page, D)
    if case["op"] == "attn":
        st.scale = D ** -0.5
        st.masks = torch.tensor(_masks(case["new"]), dtype=torch.int64, device="cuda") if case["tree"] else None
        st.out = torch.zeros((T, H * D), dtype=dt, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------- plain forms
def _rope(x, st, weight, bias):
    """Norm and rotation of x [T, heads, D]: 32 bits."""
    case, x = st.case, x.float()
    if case["norm"] == "rms":
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    elif case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        if bias is not None:
            x = x + bias.float()
    rot = case["rot"]
    half = rot // 2
    cs = st.cos_sin[st.position.long()]
    c, s = cs[:, None, :half], cs[:, None, half:]
    y = x.clone()
    a = x[..., 0:rot:2] if case["interleaved"] else x[..., :half]
    b = x[..., 1:rot:2] if case["interleaved"] else x[..., half:rot]
    if case["interleaved"]:
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        y[..., :half], y[..., half:rot] = a * c - b * s, b * c + a * s
    return y


def _owner(st):
    """Stream and index inside it of every row that belongs to one."""
    t = torch.arange(st.rows, device="cuda", dtype=torch.int32)
    s = torch.searchsorted(st.row_begin, t, right=True) - 1
    return s, t - st.row_begin[s]


def _plain_norm_rope(st):
    st.q_out.copy_(_rope(st.q, st, st.q_weight, st.q_bias))
    st.k_out.copy_(_rope(st.k, st, st.k_weight, st.k_bias))
    return st.q_out, st.k_out


def _plain_append(st):
    n, page = st.rows, st.case["page"]
    st.q_out[:n] = _rope(st.q, st, st.q_weight, st.q_bias)[:n].to(st.q_out.dtype)
    s, i = _owner(st)
    at = (st.kv_len[s] - (st.row_begin[s + 1] - st.row_begin[s]) + i).long()
    to = st.block_table[s, at // page].long()
    st.k_pages[to, :, at % page] = _rope(st.k, st, st.k_weight, st.k_bias)[:n].to(st.k_pages.dtype)
    st.v_pages[to, :, at % page] = st.v[:n]
    return st.q_out, st.k_pages, st.v_pages


def _plain_attn(st):
    case = st.case
    S, N, H, Hkv, D = case["streams"], case["new"], case["heads"], case["kv_heads"], case["dim"]
    G, table = H // Hkv, st.block_table.long()
    keys = st.k_pages[table].transpose(1, 2).reshape(S, Hkv, -1, D).float()
    values = st.v_pages[table].transpose(1, 2).reshape(S, Hkv, -1, D).float()
    L = keys.shape[2]
    n = (st.row_begin[1:] - st.row_begin[:-1])[:, None]
    i = torch.arange(N, device="cuda")[None, :]
    rows = (st.row_begin[:-1, None] + i).clamp_max(st.q.shape[0] - 1).long()
    q = st.q[rows].float().reshape(S, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * N, D)
    j = torch.arange(L, device="cuda")[None, None, :]
    prefix = (st.kv_len[:, None] - n)[:, :, None]
    if case["tree"]:
        rel = (j - prefix).clamp(0, 63)
        seen = (j < prefix) | ((j - prefix < N) & ((st.masks[None, :, None] >> rel) & 1).bool())
    else:
        seen = j <= prefix + i[:, :, None]
    e = (q @ keys.transpose(2, 3)).reshape(S, Hkv, G, N, L).mul_(st.scale)
    e.masked_fill_(~seen[:, None, None], -math.inf)
    e.sub_(e.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e.reshape(S, Hkv, G * N, L) @ values).reshape(S, Hkv, G, N, D) / total.clamp_min(1e-38)
    o = o.permute(0, 3, 1, 2, 4).reshape(S, N, H * D)
    s, at = _owner(st)
    st.out[:st.rows] = o[s, at].to(st.out.dtype)
    return st.out


def run(st):
    op = st.case["op"]
    if not own:
        return _plain_norm_rope(st) if op == "norm_rope" else _plain_append(st) if op == "append" else _plain_attn(st)
    import paper_2510_25739_b200 as hawk
    case = st.case
    if op == "attn":
        return hawk.paged_attn(st.q, st.k_pages, st.v_pages, st.block_table, st.row_begin, st.kv_len, case["new"], case["kv"], st.scale,
                               anc_mask=st.masks, out=st.out)
    norm = dict(norm=case["norm"], eps=EPS, q_weight=st.q_weight, k_weight=st.k_weight, q_bias=st.q_bias, k_bias=st.k_bias,
                interleaved=case["interleaved"], q_out=st.q_out)
    if op == "norm_rope":
        return hawk.qk_norm_rope(st.q, st.k, st.position, st.cos_sin, k_out=st.k_out, **norm)
    q_out = hawk.rope_append(st.q, st.k, st.v, st.position, st.cos_sin, st.k_pages, st.v_pages, st.block_table, st.row_begin,
                             st.kv_len, **norm)
    return q_out, st.k_pages, st.v_pages


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    ns, ls = _lengths(case)
    H, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
    rows = sum(ns)
    if case["op"] == "attn":
        pairs = sum(n * (l - n) + n * (n + 1) // 2 for n, l in zip(ns, ls))
        if case["tree"]:
            pairs = sum(n * (l - n) for n, l in zip(ns, ls)) + len(ns) * sum(bin(m).count("1") for m in _masks(case["new"]))
        read = sum(l for n, l in zip(ns, ls) if n)
        return {"bytes": 4.0 * read * Hkv * D + 4.0 * rows * H * D, "flops": 4.0 * D * H * pairs}
    if case["op"] == "norm_rope":
        rows += SPARE_ROWS if case["ragged"] else 0
    heads = H + Hkv if case["op"] == "norm_rope" else H + 2 * Hkv
    table = min(rows, case["kv"] + 1) * case["rot"] * 4.0
    return {"bytes": 4.0 * rows * heads * D + table, "flops": 10.0 * rows * (H + Hkv) * D}


# ---------------------------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_head_rows(x, case, weight, bias, cs):
    """One head after another of x [rows, heads, D]; cs [rows, rot] holds cos | sin."""
    x, out = x.double(), []
    for h in range(x.shape[1]):
        y = x[:, h]
        w = None if weight is None else (weight[h] if weight.dim() == 2 else weight).double()
        b = None if bias is None else (bias[h] if bias.dim() == 2 else bias).double()
        if case["norm"] == "layer":
            mean = y.sum(1, keepdim=True) / y.shape[1]
            y = (y - mean) / ((y - mean).pow(2).sum(1, keepdim=True) / y.shape[1] + EPS).sqrt() * w
            y = y if b is None else y + b
        elif case["norm"] == "rms":
            y = y / (y.pow(2).sum(1, keepdim=True) / y.shape[1] + EPS).sqrt() * w
        half = case["rot"] // 2
        turned = torch.view_as_complex(torch.stack([cs[:, :half], cs[:, half:]], -1).double().contiguous())
        if case["interleaved"]:
            z = torch.view_as_complex(y[:, :2 * half].reshape(-1, half, 2).contiguous()) * turned
            first = torch.view_as_real(z).reshape(-1, 2 * half)
        else:
            z = torch.complex(y[:, :half].contiguous(), y[:, half:2 * half].contiguous()) * turned
            first = torch.cat([z.real, z.imag], 1)
        out.append(torch.cat([first, y[:, 2 * half:]], 1))
    return torch.stack(out, 1)


def exact(case, seed):
    st = prepare(case, seed)
    begin, lens = st.row_begin.tolist(), st.kv_len.tolist()
    if case["op"] != "attn":
        cs = st.cos_sin[st.position.long()]
        q = _exact_head_rows(st.q, case, st.q_weight, st.q_bias, cs)
        k = _exact_head_rows(st.k, case, st.k_weight, st.k_bias, cs)
        if case["op"] == "norm_rope":
            return q, k
        q[st.rows:] = 0
        kp, vp = st.k_pages.double(), st.v_pages.double()
        table = st.block_table.tolist()
        for s in range(case["streams"]):
            n = begin[s + 1] - begin[s]
            first, at = lens[s] - n, begin[s]
            while n > 0:  # page by page
                off = first % case["page"]
                count, to = min(case["page"] - off, n), table[s][first // case["page"]]
                kp[to, :, off:off + count] = k[at:at + count].transpose(0, 1)
                vp[to, :, off:off + count] = st.v[at:at + count].double().transpose(0, 1)
                first, at, n = first + count, at + count, n - count
        return q, kp, vp
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(st.out.shape, dtype=torch.float64, device="cuda").reshape(-1, H, D)
    for s in range(case["streams"]):
        n, l = begin[s + 1] - begin[s], lens[s]
        if not n:
            continue
        pages = st.block_table[s, :-(-l // page)].long()
        hidden = torch.arange(l, device="cuda")[None, :] > torch.arange(l - n, l, device="cuda")[:, None]
        if case["tree"]:
            hidden[:, l - n:] = torch.tensor([[not m >> c & 1 for c in range(n)] for m in _masks(case["new"])[:n]], device="cuda")
        for hk in range(Hkv):
            keys = st.k_pages[pages, hk].reshape(-1, D)[:l].double()
            values = st.v_pages[pages, hk].reshape(-1, D)[:l].double()
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                e = st.q[begin[s]:begin[s + 1], h].double() @ keys.T * st.scale
                out[begin[s]:begin[s + 1], h] = torch.softmax(e.masked_fill(hidden, -math.inf), 1) @ values
    return out.reshape(-1, H * D)
