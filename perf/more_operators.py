"""Measured cases of what a serving loop does between two verify steps.

Five operators, one `run` each:
  sample   sample: one token a row from its logits (guidance, temperature, top-k, top-p, min-p) and a given random number
  grow     pages_resize, then pages_copy: streams of a paged cache grow, are cut or freed; a shared page that is written is copied first
  fork     pages_fork: streams continue others (several images of a prompt, reordered batches), pages shared by reference
  compact  pages_compact, then pages_copy: used pages move to the lowest ids
  keep     pages_keep: the rows of an accepted path move to the front of their block

The cache's state is a block table (page ids of every stream), the streams' lengths in keys and a count of table entries for each
page; a page without any is free.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _sample(name, dtype, rows, vocab, guided=False, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0, per_row=False, probs=False, begin=0,
            end=None, std=2.5):
    return dict(name=name, op="sample", dtype=dtype, rows=rows, vocab=vocab, begin=begin, end=vocab if end is None else end,
                guided=guided, top_k=top_k, top_p=top_p, min_p=min_p, temperature=temperature, per_row=per_row, probs=probs, std=std)


def _cache(name, op, dtype, streams, kv, page, kv_heads, dim, layers, share=1, new=1, spare=8, nodes=0, moves=0):
    return dict(name=name, op=op, dtype=dtype, streams=streams, kv=kv, page=page, kv_heads=kv_heads, dim=dim, layers=layers, share=share,
                new=new, spare=spare, nodes=nodes, moves=moves)


def listed():
    return [
        # the first image token of one sequence (two guidance rows), the smallest call
        _sample("sample_first_token", "fp32", 1, 16384, guided=True, top_k=2000),
        # a batch whose requests bring settings of their own, two guidance rows each
        _sample("sample_batch_settings", "fp32", 64, 16384, guided=True, per_row=True),
        # text of a model with a long, odd vocabulary, logits in bf16 (many ties)
        _sample("sample_text_odd", "bf16", 48, 100003, top_p=0.9, min_p=0.01, temperature=0.8),
        # drafts of a full batch (64 x 8) with the distributions that the verification reads
        _sample("sample_drafts_probs", "fp32", 512, 16384, top_p=0.95, probs=True),
        # one token more for one sequence (two guidance streams)
        _cache("grow_decode_tiny", "grow", "bf16", 2, 128, 16, 16, 64, 1),
        # 32 prompts, eight images of each: those just forked copy the page they begin to write
        _cache("grow_forked_batch", "grow", "bf16", 256, 1149, 16, 20, 64, 4, share=8, new=8, spare=64),
        # images of a few prompts join a small batch
        _cache("fork_small", "fork", "bf16", 16, 1149, 16, 20, 64, 1, share=4),
        # a large batch over long caches is reordered
        _cache("fork_reorder_long", "fork", "bf16", 512, 9001, 16, 8, 128, 1, share=8),
        # trees of 22 nodes at the XL shape, eight sequences
        _cache("keep_tree_xl", "keep", "bf16", 16, 1171, 16, 20, 64, 12, nodes=22),
        # trees of 64 nodes, a full batch
        _cache("keep_tree_stress", "keep", "bf16", 128, 543, 32, 20, 64, 4, nodes=64),
        # a small pool gives up a few pages
        _cache("compact_small", "compact", "fp16", 12, 701, 24, 8, 128, 2, spare=300, moves=16),
        # a large, sparse pool is packed
        _cache("compact_large", "compact", "bf16", 128, 1149, 16, 20, 64, 1, share=2, spare=9000, moves=4096),
    ]


MOST_BYTES = 1.6e9  # of a cache's pages


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("sample", "sample", "grow", "fork", "keep", "compact"))
    if op == "sample":
        vocab = log(40, 200000)
        rows = log(1, max(1, min(600, 512 * 16384 // vocab)))
        begin = rng.choice((0, 0, rng.randrange(0, vocab // 3)))
        case = _sample("", rng.choice(("fp32", "fp32", "bf16", "fp16")), rows, vocab, guided=rng.random() < 0.5,
                       top_k=rng.choice((0, 0, 1, log(1, 3000))), top_p=rng.choice((1.0, 0.9, round(rng.uniform(0.05, 0.999), 3))),
                       min_p=rng.choice((0.0, 0.0, 0.02, round(rng.uniform(0.001, 0.5), 3))),
                       temperature=rng.choice((1.0, 0.0, round(rng.uniform(0.3, 1.8), 2), round(rng.uniform(0.3, 1.8), 2))),
                       per_row=rng.random() < 0.4, probs=rng.random() < 0.3, begin=begin,
                       end=rng.choice((vocab, rng.randint(begin + 1, vocab))), std=round(rng.uniform(0.5, 5.0), 2))
        del case["name"]
        return case
    dim, page = rng.choice((64, 128)), rng.choice((8, 16, 16, 24, 32, 64, 128))
    heads, layers = rng.choice((1, 2, 4, 8, 16, 20, 32)), 1 if op == "fork" else log(1, 12)
    kv = log(1, 9000 if op == "fork" else 3500)
    nodes = min(kv, rng.randint(2, 64)) if op == "keep" else 0
    share = rng.choice((1, 2, 4, 8))
    if op == "keep":
        share = 1
    row = 4.0 * heads * dim * layers
    most = 512 if op == "fork" else int(max(2, min(256, MOST_BYTES / 2 / (row * (kv + page)))))
    streams = 2 * log(1, max(1, most // 2))
    spare = log(1, 64) if op != "compact" else log(4, max(8, min(9000, int(MOST_BYTES / 2 / (row * page)))))
    case = _cache("", op, rng.choice(("bf16", "fp16")), streams, kv, page, heads, dim, layers, share=share, new=log(1, 70), spare=spare,
                  nodes=nodes, moves=log(1, 4096) if op == "compact" else 0)
    del case["name"]
    return case


class State:
    pass


def _prepare_sample(st, case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    R, V = case["rows"], case["vocab"]
    x = torch.empty((R * (2 if case["guided"] else 1), V), dtype=torch.float32, device="cuda").normal_(0.0, case["std"], generator=g)
    if case["guided"]:  # the unconditional row is near the conditional one
        x[R:] = 0.9 * x[:R] + 0.1 * x[R:]
    x[torch.rand(x.shape, generator=g, device="cuda") < 0.01] = -math.inf  # ids that a grammar or a mask forbids
    st.logits = x.to(DTYPES[case["dtype"]])
    st.u = torch.rand(R, generator=g, device="cuda")
    st.scale = 3.0 if case["guided"] else None
    st.temperature, st.top_k, st.top_p, st.min_p = case["temperature"], case["top_k"], case["top_p"], case["min_p"]
    if case["per_row"]:
        def some(values, dtype=torch.float32):
            at = torch.randint(len(values), (R,), generator=g, device="cuda")
            return torch.tensor(values, dtype=dtype, device="cuda")[at]
        st.temperature, st.top_k = some([0.0, 0.7, 0.9, 1.0, 1.0, 1.3]), some([0, 0, 1, 50, 1000, 2000], torch.int32)
        st.top_p, st.min_p = some([1.0, 0.5, 0.9, 0.95, 0.99]), some([0.0, 0.0, 0.01, 0.1])
        if case["guided"]:
            st.scale = some([1.0, 3.0, 4.0, 7.5])
    st.token = torch.zeros(R, dtype=torch.int32, device="cuda")
    st.token_prob = torch.zeros(R, device="cuda")
    st.probs = torch.zeros((R, V), device="cuda") if case["probs"] else None


def _layout(case, seed):
    """Lengths, block table and reference counts of a cache in use, on the host.  Streams in groups of `share` have a prompt's pages in
    common; one that is just forked (a third of them) shares the page that it will write next as well.  Every seed has the same
    lengths, and what the streams do next; which pages they have goes by the seed."""
    r = np.random.RandomState(case["streams"] * 7919 + case["kv"] * 31 + case["page"])
    S, page, share = case["streams"], case["page"], case["share"]
    least = max(case["nodes"], 1, case["kv"] // 2)
    prompt = [int(r.randint(least, case["kv"] + 1)) for _ in range(-(-S // share))]
    prompt[r.randint(len(prompt))] = case["kv"]
    lens, width = [], -(-(case["kv"] + case["new"]) // page)
    table = np.zeros((S, width), np.int64)
    made = 0
    tail = {}
    for s in range(S):
        p = prompt[s // share]
        first = s % share == 0
        grown = 0 if first or r.rand() < 1 / 3 else int(r.randint(0, case["kv"] - p + 1))
        lens.append(p + grown)
        full, need = p // page, -(-(p + grown) // page)
        if first:
            table[s, :need] = made + np.arange(need)
            made += need
            tail[s // share] = s
        else:
            shared = need if grown == 0 else full
            table[s, :shared] = table[tail[s // share], :shared]
            table[s, shared:need] = made + np.arange(need - shared)
            made += need - shared
    n_pages = made + case["spare"]
    if case["op"] == "grow":  # room for the growth and the copies
        n_pages += S * (-(-case["new"] // page) + 2)
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages)
    lens = np.array(lens, np.int64)
    used = np.arange(width)[None, :] < -(-lens // page)[:, None]
    table = np.where(used, order[table], 0)
    refs = np.bincount(table[used], minlength=n_pages)
    return r, lens, table, refs


def _new_lengths(r, case, lens):
    S = case["streams"]
    what = r.rand(S)
    new = np.where(what < 0.8, lens + r.randint(1, case["new"] + 1, S), lens)               # some are idle,
    new = np.where((what >= 0.88) & (what < 0.96), np.maximum(lens - case["new"], 0), new)  # cut behind what was accepted,
    return np.where(what >= 0.96, 0, new)                                                   # finished


def _tree_paths(r, B, nodes):
    """An accepted path in a random candidate tree of each sequence: nodes in order, -1 behind the last."""
    paths, accepted = np.full((B, 12), -1, np.int64), np.zeros(B, np.int64)
    parent = [-1] + [int(r.randint(max(0, (i - 1) // 3), i)) for i in range(1, nodes)]
    for b in range(B):
        chain, at = [], int(r.randint(nodes))
        while at > 0:
            chain.append(at)
            at = parent[at]
        chain = chain[::-1][:12]
        paths[b, :len(chain)] = chain
        accepted[b] = len(chain)
    return paths, accepted


def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _prepare_cache(st, case, seed):
    r, lens, table, refs = _layout(case, seed)
    S, op = case["streams"], case["op"]
    st.page, st.n_pages = case["page"], len(refs)
    st.block_table, st.kv_len, st.page_refs = _int(table), _int(lens), _int(refs)
    if op != "fork":
        g = torch.Generator(device="cuda").manual_seed(int(seed))
        shape = (case["layers"], st.n_pages, case["kv_heads"], case["page"], case["dim"])
        st.k_pages, st.v_pages = (torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g) for _ in range(2))
    if op == "grow":
        st.new_len = _int(_new_lengths(r, case, lens))
    if op == "fork":
        parent = r.randint(0, S, S)
        stay = r.rand(S) < 0.4
        parent = np.where(stay, np.arange(S), parent)
        parent[r.rand(S) < 0.05] = -1  # freed
        st.parent = _int(parent)
        kept = np.where(parent >= 0, lens[np.maximum(parent, 0)], 0)
        st.length = _int(np.where(r.rand(S) < 0.2, kept // 2, kept))  # some take a part only, as of a prompt
    if op == "keep":
        n = case["nodes"]
        st.row_begin = _int(np.arange(S + 1) * n)
        path, accepted = _tree_paths(r, S // 2, n)
        st.path, st.accept_len = _int(path), _int(accepted)
    st.out_table, st.out_len, st.out_refs = st.block_table.clone(), torch.zeros_like(st.kv_len), torch.zeros_like(st.page_refs)
    st.copies = torch.zeros((case["moves"] if op == "compact" else S, 3), dtype=torch.int32, device="cuda")
    st.top = torch.zeros(1, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    st = State()
    st.case = case
    (_prepare_sample if case["op"] == "sample" else _prepare_cache)(st, case, int(seed))
    return st


# ---------------------------------------------------------------------------------------------- plain forms
def _column(v, R):  # a setting is a 32-bit number, whether it comes for all rows or for each
    return v.double()[:, None] if torch.is_tensor(v) else torch.full((R, 1), float(v), device="cuda").double()


def _plain_sample(st):
    case, R = st.case, st.case["rows"]
    x = st.logits[:, case["begin"]:case["end"]].float()
    if case["guided"]:  # the guided logit is a 32-bit number, and the rest goes by its value
        c, n = x[:R], x[R:]
        x = (n.double() + _column(st.scale, R) * (c - n).double()).float()
        x = x.masked_fill((c == -math.inf) | (n == -math.inf), -math.inf)
    x = x.masked_fill(x.isnan() | (x == math.inf), -math.inf).double()
    n = x.shape[1]
    T, k, p, least = (_column(v, R) for v in (st.temperature, st.top_k, st.top_p, st.min_p))
    ids = torch.arange(n, device="cuda")[None, :]
    top = x.amax(1, keepdim=True)
    greedy = T == 0
    z = torch.where(greedy, torch.zeros_like(x).masked_fill(x != top, -math.inf), (x - top) / torch.where(greedy, 1.0, T))
    first = torch.where(x == top, ids, n).amin(1, keepdim=True)
    z = z.masked_fill(greedy & (ids != first), -math.inf)
    order, at = x.sort(1, descending=True)
    kth = order.gather(1, (k.long() - 1).clamp(0, n - 1))
    kept = (x >= kth) | (k <= 0) | (k > n)
    w = torch.where(kept & (x > -math.inf), z.exp(), 0.0)
    run = w.gather(1, at).cumsum(1)
    need = (run < p * run[:, -1:]).sum(1, keepdim=True).clamp(max=n - 1)
    kept = (x >= order.gather(1, need)) | (p >= 1)
    kept &= (z >= least.log()) | (least <= 0)
    w = torch.where(kept, w, 0.0)
    run = w.cumsum(1)
    total = run[:, -1:]
    pick = (run <= st.u.double()[:, None] * total).sum(1, keepdim=True).clamp(max=n - 1)
    some = top > -math.inf
    probs = torch.where(some, w / total, 0.0)
    st.token[:] = torch.where(some, pick + case["begin"], -1)[:, 0]
    st.token_prob[:] = probs.gather(1, pick)[:, 0]
    if st.probs is not None:
        st.probs.zero_()
        st.probs[:, case["begin"]:case["end"]] = probs
    return [st.token, st.token_prob] + ([st.probs] if case["probs"] else [])


def _pages_of(keys, page):
    return (keys + page - 1) // page


def _plain_copy(st):
    """Rows [0, rows) of the pages `src` to the pages `dst`, all layers: entries without a copy write a page to itself."""
    src, dst, rows = st.copies.long().unbind(1)
    some = src >= 0
    to = torch.where(some, dst, st.spot)
    keep = (torch.arange(st.page, device="cuda")[None, :] < rows[:, None]) & some[:, None]
    for x in (st.k_pages, st.v_pages):
        x[:, to] = torch.where(keep[None, :, None, :, None], x[:, src.clamp(min=0)], x[:, to])


def _plain_grow(st):
    table, page = st.block_table.long(), st.page
    S, W = table.shape
    old, new = st.kv_len.long(), st.new_len.long()
    have, want = _pages_of(old, page), _pages_of(new, page)
    j = torch.arange(W, device="cuda")[None, :]
    refs = st.page_refs.long()
    gone = (j >= want[:, None]) & (j < have[:, None])
    refs = refs.scatter_add(0, table.flatten(), -gone.long().flatten())
    last = table.gather(1, (have - 1).clamp(min=0)[:, None])[:, 0]
    own_copy = (new > old) & (old % page != 0) & (refs[last] > 1)
    need = torch.where(new > old, want - have + own_copy.long(), 0)
    free = torch.sort((refs > 0).long(), stable=True)
    end = need.cumsum(0)
    served = (need == 0) | (end <= (free.values == 0).sum())
    own_copy &= served
    rank = j - have[:, None] + own_copy.long()[:, None]
    fresh = (rank >= 0) & (j < want[:, None]) & (served & (need > 0))[:, None]
    page_at = free.indices[(end[:, None] - need[:, None] + rank).clamp(0, len(refs) - 1)]
    out = torch.where(fresh, page_at, table)
    refs = refs.scatter_add(0, page_at.flatten(), fresh.long().flatten())
    refs = refs.scatter_add(0, last, -own_copy.long())
    st.out_table.copy_(torch.where(j < torch.where(served, want, have)[:, None], out, table))
    st.out_len.copy_(torch.where(served, new, old))
    st.out_refs.copy_(refs)
    none = torch.full_like(last, -1)
    copy = torch.stack([torch.where(own_copy, last, none), torch.where(own_copy, out.gather(1, (have - 1).clamp(min=0)[:, None])[:, 0], none),
                        torch.where(own_copy, old % page, 0)], 1)
    st.copies.copy_(copy)
    st.spot = free.indices[-1]  # a page in use: what is written there is what it held
    _plain_copy(st)
    return st.out_table, st.out_len, st.out_refs, st.copies, st.k_pages, st.v_pages


def _plain_fork(st):
    table, page = st.block_table.long(), st.page
    S, W = table.shape
    j = torch.arange(W, device="cuda")[None, :]
    parent = st.parent.long()
    new = torch.where(parent >= 0, torch.minimum(st.length, st.kv_len[parent.clamp(min=0)]), 0)
    held, takes = j < _pages_of(st.kv_len, page)[:, None], j < _pages_of(new, page)[:, None]
    rows = table[parent.clamp(min=0)]
    refs = st.page_refs.long().scatter_add(0, table.flatten(), -held.long().flatten())
    st.out_refs.copy_(refs.scatter_add(0, rows.flatten(), takes.long().flatten()))
    st.out_table.copy_(torch.where(takes, rows, st.out_table))
    st.out_len.copy_(new)
    return st.out_table, st.out_len, st.out_refs


def _plain_compact(st):
    refs, M = st.page_refs.long(), st.copies.shape[0]
    n = len(refs)
    order = torch.sort((refs > 0).long(), stable=True).indices  # free pages, then pages in use, ascending
    free = (refs == 0).sum()
    i = torch.arange(M, device="cuda")
    to, frm = order[i.clamp(max=n - 1)], order[(n - 1 - i).clamp(min=0)]
    moved = (i < free) & (i < n - free) & (to < frm)
    where = torch.arange(n + 1, device="cuda")
    where = where.scatter(0, torch.where(moved, frm, n), torch.where(moved, to, n))[:n]
    table = st.block_table.long()
    used = torch.arange(table.shape[1], device="cuda")[None, :] < _pages_of(st.kv_len, st.page)[:, None]
    st.out_table.copy_(torch.where(used, where[table], table))
    out = torch.zeros_like(refs).scatter(0, where, refs, reduce="add")
    st.out_refs.copy_(out)
    st.top.copy_(torch.where(out > 0, torch.arange(1, n + 1, device="cuda"), 0).amax()[None])
    st.copies.copy_(torch.where(moved[:, None], torch.stack([frm, to, torch.full_like(to, st.page)], 1),
                                torch.tensor([-1, -1, 0], device="cuda")[None, :]))
    st.spot = order[-1]
    _plain_copy(st)
    return st.out_table, st.out_refs, st.copies, st.top, st.k_pages, st.v_pages


def _plain_keep(st):
    S, page = st.case["streams"], st.page
    n = (st.row_begin[1:] - st.row_begin[:-1]).long()
    path = st.path.long().repeat(S // st.path.shape[0], 1)
    accepted = st.accept_len.long().repeat(S // st.path.shape[0])
    i = torch.arange(path.shape[1], device="cuda")[None, :]
    base = (st.kv_len.long() - n)[:, None]
    live = i < accepted[:, None]
    to = base + 1 + torch.where(live, i, 0)
    frm = torch.where(live, base + path, to)
    frm = torch.where(live | (accepted[:, None] == 0), frm, base + path[:, :1])  # places that are not live write what the first one does
    table = st.block_table.long()
    rows = [(table.gather(1, a // page), a % page) for a in (frm, to)]
    for x in (st.k_pages, st.v_pages):
        x[:, rows[1][0], :, rows[1][1]] = x[:, rows[0][0], :, rows[0][1]]
    st.out_len.copy_(base[:, 0] + torch.minimum(n, 1 + accepted))
    return st.out_len, st.k_pages, st.v_pages


def run(st):
    op = st.case["op"]
    if not own:
        return {"sample": _plain_sample, "grow": _plain_grow, "fork": _plain_fork, "compact": _plain_compact, "keep": _plain_keep}[op](st)
    import paper_2510_25739_b200 as hawk
    if op == "sample":
        hawk.sample(st.logits, st.u, temperature=st.temperature, top_k=st.top_k, top_p=st.top_p, min_p=st.min_p, cfg_scale=st.scale,
                    v_begin=st.case["begin"], v_end=st.case["end"], token=st.token, token_prob=st.token_prob, probs=st.probs)
        return [st.token, st.token_prob] + ([st.probs] if st.case["probs"] else [])
    if op == "grow":
        hawk.pages_resize(st.block_table, st.kv_len, st.new_len, st.page_refs, st.page, out_table=st.out_table, out_len=st.out_len,
                          out_refs=st.out_refs, copies=st.copies)
        hawk.pages_copy(st.k_pages, st.v_pages, st.copies)
        return st.out_table, st.out_len, st.out_refs, st.copies, st.k_pages, st.v_pages
    if op == "fork":
        hawk.pages_fork(st.block_table, st.kv_len, st.parent, st.page_refs, st.page, length=st.length, out_table=st.out_table,
                        out_len=st.out_len, out_refs=st.out_refs)
        return st.out_table, st.out_len, st.out_refs
    if op == "compact":
        hawk.pages_compact(st.block_table, st.kv_len, st.page_refs, st.page, st.copies.shape[0], out_table=st.out_table,
                           out_refs=st.out_refs, copies=st.copies, top=st.top)
        hawk.pages_copy(st.k_pages, st.v_pages, st.copies)
        return st.out_table, st.out_refs, st.copies, st.top, st.k_pages, st.v_pages
    hawk.pages_keep(st.k_pages, st.v_pages, st.block_table, st.row_begin, st.kv_len, st.path, st.accept_len, out_len=st.out_len)
    return st.out_len, st.k_pages, st.v_pages


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        R, n = case["rows"], case["end"] - case["begin"]
        size = 4.0 if case["dtype"] == "fp32" else 2.0
        return {"bytes": R * n * size * (2 if case["guided"] else 1) + (4.0 * R * case["vocab"] if case["probs"] else 0) + 12.0 * R,
                "flops": 10.0 * R * n}
    r, lens, table, refs = _layout(case, 1)
    S, page = case["streams"], case["page"]
    row = 4.0 * case["kv_heads"] * case["dim"] * case["layers"]  # a key and a value in all layers
    entries = float((-(-lens // page)).sum())
    if case["op"] == "fork":  # entries read for the counts, read and written for the children; counts read and written
        return {"bytes": 12.0 * entries + 8.0 * len(refs) + 16.0 * S, "flops": 2.0 * entries}
    if case["op"] == "keep":
        paths, accepted = _tree_paths(r, S // 2, case["nodes"])
        moved = 2.0 * float(accepted.sum())
        return {"bytes": 2.0 * row * moved + 4.0 * paths.size + 16.0 * S, "flops": 2.0 * S}
    if case["op"] == "grow":
        new = _new_lengths(r, case, lens)
        shared = (refs[table[np.arange(S), np.maximum(-(-lens // page) - 1, 0)]] > 1) & (new > lens)
        rows = float(((lens % page) * shared).sum())  # (some cuts may leave a page to one stream, which then need not copy it)
        return {"bytes": 2.0 * row * rows + 8.0 * len(refs) + 24.0 * S, "flops": 2.0 * len(refs)}
    used = int((refs > 0).sum())
    moved = min(case["moves"], int((refs[used:] > 0).sum()))
    return {"bytes": 2.0 * row * page * moved + 8.0 * len(refs) + 8.0 * entries, "flops": 2.0 * len(refs)}


# ---------------------------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_row(x, T, k, p, least, u):
    """(id, probabilities) of one row of logits (float64, -inf: never), by distinct values from the largest down."""
    n = len(x)
    if not np.isfinite(x).any():
        return -1, np.zeros(n)
    top = x.max()
    if T == 0:
        at = int(np.flatnonzero(x == top)[0])
        probs = np.zeros(n)
        probs[at] = 1.0
        return at, probs
    values, place, count = np.unique(-x[np.isfinite(x)], return_inverse=True, return_counts=True)
    values = -values
    weight = np.exp((values - top) / T)
    if 0 < k < n:
        reached = np.flatnonzero(np.cumsum(count) >= k)
        if len(reached):
            weight[reached[0] + 1:] = 0
    if p < 1:
        mass = np.cumsum(weight * count)
        weight[np.flatnonzero(mass >= p * mass[-1])[0] + 1:] = 0
    if least > 0:
        weight[(values - top) / T < math.log(least)] = 0
    probs = np.zeros(n)
    probs[np.isfinite(x)] = weight[place]
    run = np.cumsum(probs)
    at = int(np.searchsorted(run, u * run[-1], side="right"))
    return min(at, n - 1), probs / run[-1]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "fork":
        return None  # whole numbers only
    if case["op"] != "sample":
        if case["op"] == "grow":
            table, page = st.block_table.tolist(), case["page"]
            refs, copies = st.page_refs.tolist(), []
            steps = list(zip(st.kv_len.tolist(), st.new_len.tolist()))
            for s, (old, new) in enumerate(steps):
                for j in range(-(-new // page), -(-old // page)):
                    refs[table[s][j]] -= 1
            free = iter([i for i, c in enumerate(refs) if c == 0])
            for s, (old, new) in enumerate(steps):
                if new > old:
                    if old % page and refs[table[s][old // page]] > 1:
                        copies.append((table[s][old // page], next(free), old % page))
                    for _ in range(-(-old // page), -(-new // page)):
                        next(free)
            before = [None] * 4
        elif case["op"] == "compact":
            refs = st.page_refs.tolist()
            free, used = [i for i, c in enumerate(refs) if not c], [i for i, c in enumerate(refs) if c][::-1]
            copies = [(a, b, case["page"]) for a, b in list(zip(used, free))[:case["moves"]] if b < a]
            before = [None] * 4
        k, v = st.k_pages.double(), st.v_pages.double()
        if case["op"] == "keep":
            S, n, page = case["streams"], case["nodes"], case["page"]
            table, lens, paths, accepted = (t.tolist() for t in (st.block_table, st.kv_len, st.path, st.accept_len))
            for s in range(S):
                for i in range(accepted[s % (S // 2)]):
                    a, b = lens[s] - n + paths[s % (S // 2)][i], lens[s] - n + 1 + i
                    for x in (k, v):
                        x[:, table[s][b // page], :, b % page] = x[:, table[s][a // page], :, a % page]
            return [None, k, v]
        for a, b, rows in copies:
            for x in (k, v):
                x[:, b, :, :rows] = x[:, a, :, :rows]
        return before + [k, v]
    R = case["rows"]
    x = st.logits[:, case["begin"]:case["end"]].float().cpu().numpy()

    def each(v):
        return v.double().cpu().numpy() if torch.is_tensor(v) else np.full(R, np.float32(v)).astype(np.float64)

    if case["guided"]:  # subtract, then multiply and add, each rounded to 32 bits
        with np.errstate(invalid="ignore"):
            wide = x[R:].astype(np.float64) + each(st.scale)[:, None] * (x[:R] - x[R:]).astype(np.float64)
        x = np.where(np.isneginf(x[:R]) | np.isneginf(x[R:]), -np.inf, wide.astype(np.float32))
    x = x.astype(np.float64)
    T, k, p, least, u = (each(v) for v in (st.temperature, st.top_k, st.top_p, st.min_p, st.u))
    chosen, probs = np.zeros(R), np.zeros((R, case["vocab"])) if case["probs"] else None
    for row in range(R):
        at, q = _exact_row(x[row], T[row], k[row], p[row], least[row], u[row])
        chosen[row] = q[at] if at >= 0 else 0.0
        if probs is not None:
            probs[row, case["begin"]:case["end"]] = q
    return [None, torch.from_numpy(chosen)] + ([torch.from_numpy(probs)] if probs is not None else [])
