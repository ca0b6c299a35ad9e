"""The calls between two verify steps together with those of a step, as a serving loop runs them: two prompts forked into guidance
streams, pages made for a tree's rows and copied where they are shared, rows appended, the tree attended to, verified against drafts that
hawk_sample drew, the accepted path kept, the rest given back, the pool packed now and then.  After every step each stream's cache
rows are, bit for bit, what was appended for it, the attention is that of the plain form over those rows, and the counts add up."""
import numpy as np
import pytest
import torch

import paper_2510_25739_b200 as hawk
from oracle import paged
from tests import _serving as sv
from tests._paged import f64, half_step

pytestmark = pytest.mark.gpu

H, H_KV, D, LAYERS = 4, 2, 64, 2
CHILDREN = [[1, 2], [3, 4], [5], [6], [], [], []]  # a tree of seven nodes
N = len(CHILDREN)


def _tree():
    """child_begin (breadth first: the children of a node follow each other), ancestor masks, depths."""
    begin, masks, depth = [1], [1], [0]
    for n, c in enumerate(CHILDREN):
        begin.append(begin[-1] + len(c))
    for n, c in enumerate(CHILDREN):
        for k in c:
            masks.append(masks[n] | 1 << k)
            depth.append(depth[n] + 1)
    return begin, masks, depth


@pytest.mark.parametrize("page", [8, 16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_loop(page, dtype):
    g = torch.Generator(device="cuda").manual_seed(page)
    B, V, n_pages, width = 3, 512, 60, 12
    S = 2 * B
    k_pages, v_pages = (torch.full((LAYERS, n_pages, H_KV, page, D), 3e4, dtype=dtype, device="cuda") for _ in range(2))
    table = torch.zeros((2, width), dtype=torch.int32, device="cuda")
    lens, refs = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    child_begin, masks, depth = _tree()
    anc = torch.tensor(masks, dtype=torch.int64, device="cuda")
    head = torch.empty((V, H * D), dtype=torch.bfloat16, device="cuda").normal_(0, 0.1, generator=g)
    mirror = [[np.zeros((LAYERS, 0, H_KV, D)) for _ in range(2)] for _ in range(2)]  # keys and values of each stream

    def rows(n):
        return [torch.empty((n, heads, D), dtype=dtype, device="cuda").normal_(generator=g) for heads in (H, H_KV, H_KV)]

    def append(begin, counts, new_len):
        q = None
        for layer in range(LAYERS):
            q, k, v = rows(sum(counts))
            q = hawk.rope_append(q, k, v, None, None, k_pages[layer], v_pages[layer], table, begin, new_len, dev_status=status)
            for s, n in enumerate(counts):
                at = sum(counts[:s])
                for which, x in enumerate((k, v)):
                    part = f64(x[at:at + n])[None]
                    mirror[s][which] = _grown(mirror[s][which], layer, part)
        return q

    def _grown(have, layer, part):
        if layer == 0:
            have = np.concatenate([have, np.zeros((LAYERS, part.shape[1], H_KV, D))], 1)
        have[layer, have.shape[1] - part.shape[1]:] = part[0]
        return have

    def check():
        torch.cuda.synchronize()
        assert int(status) == 0 and sv.check_counts(table, lens, refs, page)
        for s, n in enumerate(lens.tolist()):
            ids = table[s, :-(-n // page)].long()
            for which, pages in enumerate((k_pages, v_pages)):
                held = f64(pages[:, ids].transpose(2, 3).reshape(LAYERS, -1, H_KV, D))[:, :n]
                assert np.array_equal(held, mirror[s][which])

    # the prompts: 13 rows for the conditional streams, 5 for the unconditional ones
    prompt = torch.tensor([13, 5], dtype=torch.int32, device="cuda")
    hawk.pages_resize(table, lens, prompt, refs, page, dev_status=status)
    append(torch.tensor([0, 13, 18], dtype=torch.int32, device="cuda"), [13, 5], lens)
    check()
    table, lens = hawk.pages_fork(table, lens, torch.tensor([0] * B + [1] * B, dtype=torch.int32, device="cuda"), refs, page, dev_status=status)
    mirror = [[x.copy() for x in mirror[0 if s < B else 1]] for s in range(S)]
    check()

    row_begin = torch.arange(0, N * S + 1, N, dtype=torch.int32, device="cuda")
    node_q = torch.tensor([max(0, i - 1) for i in range(N)], dtype=torch.int32, device="cuda")
    accepted = 0
    for step in range(6):
        before = lens.clone()
        new = lens + N
        copies = hawk.pages_resize(table, lens, new, refs, page, dev_status=status)
        hawk.pages_copy(k_pages, v_pages, copies, dev_status=status)
        if step == 0:
            assert (copies[:, 0] >= 0).any()  # forked streams begin to write the prompts' last pages
        assert torch.equal(lens, new)
        q = append(row_begin, [N] * S, lens)
        check()
        out = hawk.paged_attn(q, k_pages[-1], v_pages[-1], table, row_begin, lens, N, width * page, D ** -0.5, anc_mask=anc, dev_status=status)
        want, size = paged.paged_attn(f64(q), f64(k_pages[-1]), f64(v_pages[-1]), table.cpu().numpy(), row_begin.cpu().numpy(),
                                      lens.cpu().numpy(), D ** -0.5, masks)
        h = half_step(dtype)
        assert (np.abs(f64(out).reshape(want.shape) - want) <= h * np.abs(want) + (h + 2.0 ** -11) * size).all()
        # drafts: drawn from logits near the target's, with the distributions that the verification reads
        logits = hawk.head_proj(out.bfloat16(), head).reshape(S, N, V)
        drafts = (logits[:B, :N - 1] + 0.3 * torch.empty((B, N - 1, V), device="cuda").normal_(generator=g)).reshape(-1, V)
        probs = torch.empty((B * (N - 1), V), device="cuda")
        token = hawk.sample(drafts, torch.rand(B * (N - 1), generator=g, device="cuda"), top_k=100, top_p=0.95, probs=probs, dev_status=status)
        node_token = torch.cat([torch.zeros((B, 1), dtype=torch.int32, device="cuda"), token.reshape(B, N - 1)], 1)
        n, correction, path = hawk.tree_accept(logits, probs.reshape(B, N - 1, V), node_token, node_q,
                                               torch.tensor(child_begin, dtype=torch.int32, device="cuda"),
                                               torch.rand((B, N), generator=g, device="cuda"), torch.rand((B, N), generator=g, device="cuda"),
                                               0, V, 1.5, 1.0, 100, max_depth=3, dev_status=status)
        accepted += int(n.sum())
        kept = hawk.pages_keep(k_pages, v_pages, table, row_begin, lens, path, n, dev_status=status)
        for s in range(S):
            base, chain = int(before[s]), [0] + path[s % B, :int(n[s % B])].tolist()
            mirror[s] = [np.concatenate([x[:, :base], x[:, [base + c for c in chain]]], 1) for x in mirror[s]]
            assert int(kept[s]) == base + len(chain)
        hawk.pages_resize(table, lens, kept, refs, page, dev_status=status)
        check()
        if step == 2:  # the second sequence is done; the third goes on twice
            parent = [0, 2, 2] + [B, B + 2, B + 2]
            table, lens = hawk.pages_fork(table, lens, torch.tensor(parent, dtype=torch.int32, device="cuda"), refs, page, dev_status=status)
            mirror = [[x.copy() for x in mirror[p]] for p in parent]
            check()
        if step == 4:
            top = torch.zeros(1, dtype=torch.int32, device="cuda")
            copies = hawk.pages_compact(table, lens, refs, page, n_pages, top=top, dev_status=status)
            hawk.pages_copy(k_pages, v_pages, copies, dev_status=status)
            assert int(top) == int((refs > 0).sum())
            check()
        # a plain step beside it: the token that a stream without drafts would take
        plain = hawk.sample(torch.cat([logits[:B, 0], logits[B:, 0]]), torch.rand(B, generator=g, device="cuda"), cfg_scale=1.5, top_k=100,
                            dev_status=status)
        assert ((plain >= 0) & (plain < V)).all()
    assert accepted > 0
    hawk.pages_resize(table, lens, torch.zeros_like(lens), refs, page, dev_status=status)
    assert int(status) == 0 and not refs.any() and not lens.any()
