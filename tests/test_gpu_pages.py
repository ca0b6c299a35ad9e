"""hawk_pages_* against the plain forms: growth, cuts, copies on write, forks, packing, copies in every layout, accepted paths, states that
contradict themselves, in place and not."""
import numpy as np
import pytest
import torch

import paper_2510_25739_b200 as hawk
from oracle import serving
from paper_2510_25739_b200 import binding, build
from tests import _serving as sv

pytestmark = pytest.mark.gpu


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _state(S, page, seed, share=2, longest=90, spare=60, **kw):
    r = np.random.RandomState(seed)
    lens = r.randint(0, longest + 1, S).tolist()
    width = serving.pages(longest, page) + 6
    n_pages = sum(serving.pages(n, page) for n in lens) + S * serving.pages(longest, page) // 3 + spare
    return sv.PageState(lens, page, width, n_pages, share=share, seed=seed, **kw), r


def _resize(st, new, in_place):
    table, lens, refs = st.cuda()
    status = _status()
    if in_place:
        copies = hawk.pages_resize(table, lens, sv.int32(new), refs, st.page, dev_status=status)
        return table, lens, refs, copies, int(status)
    t, n, c = torch.full_like(table, -9), torch.zeros_like(lens), torch.zeros_like(refs)
    copies = hawk.pages_resize(table, lens, sv.int32(new), refs, st.page, out_table=t, out_len=n, out_refs=c, dev_status=status)
    assert table.tolist() == st.table and lens.tolist() == st.lens and refs.tolist() == st.refs
    return t, n, c, copies, int(status)


def _same_resize(st, new, in_place):
    want_table, want_len, want_refs, want_copies, stayed = serving.resize(st.table, st.lens, new, st.refs, st.page)
    table, lens, refs, copies, status = _resize(st, new, in_place)
    assert lens.tolist() == want_len and refs.tolist() == want_refs
    assert [tuple(c) for c in copies.tolist()] == want_copies and sv.same_where_written(table, want_table)
    assert status == (binding.DEV_NO_PAGES if stayed else 0)
    return table, lens, refs


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("page", [1, 3, 16, 64])
@pytest.mark.parametrize("S", [1, 5, 64, 700])
def test_resize(S, page, in_place):
    for seed in range(3):
        st, r = _state(S, page, 10 * S + seed, share=1 + seed)
        new = [int(np.clip(n + r.choice([0, 1, -1, page, -page, 7, -7, -n, 2 * page + 1]), 0, len(st.table[0]) * page)) for n in st.lens]
        table, lens, refs = _same_resize(st, new, in_place)
        assert sv.check_counts(table, lens, refs, page)


@pytest.mark.parametrize("spare", [0, 1, 5, 17])
def test_pages_run_out(spare):
    """Streams are served in order until one does not find its pages; it and all behind it that need any stay; cuts happen all the same."""
    st = sv.PageState([30, 31, 32, 8, 20, 3], 8, 12, 0 + sum(serving.pages(n, 8) for n in (30, 31, 32, 8, 20, 3)) + spare, seed=spare)
    _same_resize(st, [33, 60, 32, 1, 41, 4], True)
    _same_resize(st, [33, 96, 32, 8, 20, 9], False)


def test_a_shared_page_is_copied_by_everyone_who_grows():
    """Eight streams share a partly filled page: four grow, one is cut inside it, one is freed, two are idle."""
    st = sv.PageState([21] * 8, 8, 6, 40, share=8, seed=1, fresh=1.0)
    new = [22, 24, 25, 40, 18, 0, 21, 21]
    table, lens, refs = _same_resize(st, new, True)
    assert refs[st.table[0][2]] == 3  # the cut one and the idle ones
    # all of them grow: the page is free behind it
    table, lens, refs = _same_resize(st, [22] * 8, True)
    assert refs[st.table[0][2]] == 0
    # a page that the other streams leave in the same call needs no copy
    _same_resize(st, [30] + [0] * 7, True)


def test_nobody_moves_and_empty_calls():
    st, _ = _state(9, 16, 3)
    table, lens, refs = _same_resize(st, list(st.lens), True)
    _same_resize(st, list(st.lens), False)
    none = sv.int32(np.zeros((0, 4)))
    hawk.pages_resize(none, none[:, 0].contiguous(), none[:, 0].contiguous(), refs, 16)
    to = torch.zeros_like(refs)
    hawk.pages_resize(none, none[:, 0].contiguous(), none[:, 0].contiguous(), refs, 16, out_refs=to)
    assert torch.equal(to, refs)


def test_the_largest_pool_and_batch():
    S, page, width, n = 4096, 4, 40, 1 << 20
    r = np.random.RandomState(2)
    st = sv.PageState(r.randint(0, 120, S).tolist(), page, width, n, share=4, seed=2)
    new = np.clip(np.array(st.lens) + r.randint(-20, 40, S), 0, width * page).tolist()
    table, lens, refs = _same_resize(st, new, True)
    st2 = type("S", (), dict(table=table.tolist(), lens=lens.tolist(), refs=refs.tolist(), page=page))
    copies, top = _compact(st2, 5000, True)[2:4]


def test_lengths_out_of_range():
    st, _ = _state(5, 8, 4)
    table, lens, refs = st.cuda()
    bad = st.lens[:]
    bad[1], bad[3] = -1, 8 * len(st.table[0]) + 1
    lens = sv.int32(bad)
    new = [n for n in st.lens]
    new[0], new[2] = -5, st.lens[2] + 3
    want = list(st.refs)
    status = _status()
    out_len = torch.zeros_like(lens)
    hawk.pages_resize(table, lens, sv.int32(new), refs, 8, out_len=out_len, dev_status=status)
    assert int(status) & binding.DEV_BAD_PREFIX
    assert out_len.tolist() == [bad[0], bad[1], new[2], bad[3], bad[4]]


def test_page_ids_out_of_range_and_counts_of_zero():
    st = sv.PageState([20, 20], 8, 4, 12, seed=5)
    for entry, new in (((0, 2), [30, 20]), ((0, 1), [0, 20])):
        for value in (-1, 12, 1 << 30):
            table, lens, refs = st.cuda()
            table[entry] = value
            status = _status()
            hawk.pages_resize(table, lens, sv.int32(new), refs, 8, dev_status=status)
            assert int(status) == binding.DEV_BAD_PAGE and lens.tolist() == new and (refs >= 0).all()
    table, lens, refs = st.cuda()
    refs[st.table[0][0]] = 0
    status = _status()
    hawk.pages_resize(table, lens, sv.int32([0, 20]), refs, 8, dev_status=status)
    assert int(status) == binding.DEV_BAD_PAGE and int(refs[st.table[0][0]]) == 0


# ------------------------------------------------------------------------------------------ fork
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S, S_out", [(1, 1), (4, 9), (9, 4), (64, 64), (300, 555)])
def test_fork(S, S_out, in_place):
    for seed, page in ((0, 16), (1, 1), (2, 5)):
        st, r = _state(S, page, 20 + seed, share=2)
        parent = np.where(r.rand(S_out) < 0.3, np.arange(S_out) % S, r.randint(-1, S, S_out)).tolist()
        for length in (None, r.randint(0, 100, S_out).tolist()):
            table, lens, refs = st.cuda()
            out_refs = None if in_place else torch.zeros_like(refs)
            status = _status()
            got_table, got_len = hawk.pages_fork(table, lens, sv.int32(parent), refs, page, length=None if length is None else sv.int32(length),
                                                 out_refs=out_refs, dev_status=status)
            want_table, want_len, want_refs = serving.fork(st.table, st.lens, parent, st.refs, page, length)
            assert int(status) == 0 and got_len.tolist() == want_len and sv.same_where_written(got_table, want_table)
            assert (refs if in_place else out_refs).tolist() == want_refs
            if not in_place:
                assert refs.tolist() == st.refs
            assert sv.check_counts(got_table, got_len, refs if in_place else out_refs, page)


def test_fork_leaves_what_it_does_not_use():
    st, _ = _state(3, 8, 30)
    table, lens, refs = st.cuda()
    out = torch.full((2, table.shape[1]), 77, dtype=torch.int32, device="cuda")
    hawk.pages_fork(table, lens, sv.int32([2, -1]), refs, 8, out_table=out)
    used = serving.pages(st.lens[2], 8)
    assert (out[0, used:] == 77).all() and (out[1] == 77).all()


def test_fork_of_bad_parents_and_lengths():
    st, _ = _state(4, 8, 31)
    for parent, length, want, flag in (([4, -2, 1, 1], None, [0, 0, st.lens[1], st.lens[1]], binding.DEV_BAD_ROWS),
                                       ([0, 1, 2, 3], [-1, 1000, 0, 1], [0, st.lens[1], 0, min(1, st.lens[3])], binding.DEV_BAD_PREFIX)):
        table, lens, refs = st.cuda()
        status = _status()
        got, n = hawk.pages_fork(table, lens, sv.int32(parent), refs, 8, length=None if length is None else sv.int32(length), dev_status=status)
        assert int(status) == flag and n.tolist() == want and sv.check_counts(got, n, refs, 8)
    table, lens, refs = st.cuda()
    with pytest.raises(binding.HawkError):
        hawk.pages_fork(table, lens, sv.int32([0, 1, 2, 3]), refs, 8, out_table=table)


# ------------------------------------------------------------------------------------------ compact
def _compact(st, moves, in_place, first=0):
    table, lens, refs = sv.int32(st.table), sv.int32(st.lens), sv.int32(st.refs)
    status, top = _status(), torch.full((1,), -5, dtype=torch.int32, device="cuda")
    out = {} if in_place else dict(out_table=torch.full_like(table, -9), out_refs=torch.zeros_like(refs))
    copies = hawk.pages_compact(table, lens, refs, st.page, moves, first_page=first, top=top, dev_status=status, **out)
    got_table, got_refs = out.get("out_table", table), out.get("out_refs", refs)
    want_table, want_refs, want_copies, want_top = serving.compact(st.table, st.lens, st.refs, st.page, moves, first)
    assert int(status) == 0 and int(top) == want_top and got_refs.tolist() == want_refs
    assert [tuple(c) for c in copies.tolist()] == want_copies and sv.same_where_written(got_table, want_table)
    return got_table, got_refs, copies, int(top)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S, page, spare", [(1, 16, 3), (6, 4, 0), (20, 8, 200), (130, 16, 5000), (3, 1, 20000)])
def test_compact(S, page, spare, in_place):
    st, _ = _state(S, page, 40 + S, spare=spare)
    for moves in (1, 7, 4096, st.n_pages + 5):
        _compact(st, moves, in_place)
    _compact(st, 50, in_place, first=min(37, st.n_pages))
    _compact(st, 50, in_place, first=st.n_pages)


def test_compact_in_steps_ends_packed():
    st, _ = _state(30, 8, 50, spare=900, held=(3, 700))
    table, lens, refs = st.cuda()
    k, v = sv.pages_tensor(0, st.n_pages, 2, 8, 16)
    before = [k[table[s, :serving.pages(n, 8)].long()].clone() for s, n in enumerate(st.lens)]
    top = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(100):
        copies = hawk.pages_compact(table, lens, refs, 8, 9, top=top)
        hawk.pages_copy(k, v, copies)
        if int(copies[0, 0]) < 0:
            break
    assert int(top) == int((refs > 0).sum()) and (refs[:int(top)] > 0).all()
    for s, n in enumerate(st.lens):
        assert torch.equal(k[table[s, :serving.pages(n, 8)].long()], before[s])


def test_compact_of_an_empty_and_a_full_pool():
    empty = sv.PageState([0, 0], 8, 4, 30)
    assert _compact(empty, 5, True)[3] == 0 and _compact(empty, 5, False, first=4)[3] == 4
    full = sv.PageState([32] * 4, 8, 4, 16, seed=3)
    assert _compact(full, 5, True)[3] == 16
    assert _compact(full, 0, True)[3] == 16


def test_compact_of_a_table_that_names_free_pages():
    """The counts say that a page is free which the table names: its id stays, whatever the workspace holds, and is flagged."""
    st = sv.PageState([32, 32], 8, 4, 60, seed=6)
    for page in (59, 58):
        if st.refs[page]:
            continue
        table, lens, refs = st.cuda()
        old = int(table[1, 3])
        table[1, 3] = page
        refs[old] = 0
        for fill in (0, 1, 255):
            ws = torch.full((hawk.pages_compact_workspace_bytes(60, 20),), fill, dtype=torch.uint8, device="cuda")
            status, out = _status(), torch.zeros_like(table)
            hawk.pages_compact(table, lens, refs, 8, 20, out_table=out, out_refs=torch.zeros_like(refs), workspace=ws, dev_status=status)
            assert int(out[1, 3]) == page and int(status) == binding.DEV_BAD_PAGE


# ------------------------------------------------------------------------------------------ copy
@pytest.mark.parametrize("layout", ["hrd", "rhd", "kv"])
@pytest.mark.parametrize("layers, H, page, D", [(0, 1, 1, 8), (1, 3, 16, 64), (3, 20, 16, 64), (2, 8, 24, 128), (1, 32, 128, 128), (2, 5, 7, 24)])
def test_copy(layers, H, page, D, layout):
    n = 13
    k, v = sv.pages_tensor(layers, n, H, page, D, torch.float16 if D == 24 else torch.bfloat16, layout, seed=D)
    want = [x.clone() for x in (k, v)]
    copies = [(3, 9, page), (4, 10, page // 2), (3, 11, 1), (-1, -1, 0), (5, 12, 0), (6, 0, page + 100), (7, 1, -3)]
    for a, b, rows in copies:
        if a >= 0:
            for x in want:
                at = (slice(None),) if layers else ()
                x[at + (b, slice(None), slice(0, max(0, rows)))] = x[at + (a, slice(None), slice(0, max(0, rows)))]
    status = _status()
    hawk.pages_copy(k, v, sv.int32(copies), dev_status=status)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and int(status) == 0


def test_copy_of_bad_pages():
    k, v = sv.pages_tensor(2, 6, 2, 8, 16)
    want = k.clone()
    want[:, 4] = want[:, 1]
    status = _status()
    hawk.pages_copy(k, v, sv.int32([(6, 2, 8), (0, 6, 8), (0, -1, 8), (1, 4, 8), (1 << 30, 1, 8)]), dev_status=status)
    assert int(status) == binding.DEV_BAD_PAGE and torch.equal(k, want)


def test_copy_past_2_31_elements():
    """Pages whose offsets pass 32 bits."""
    n, H, page, D = 600, 32, 128, 1024  # 4 M elements a page
    k = torch.zeros((n, H, page, D), dtype=torch.bfloat16, device="cuda")
    k[3] = 1.5
    k[-1] = 2.5
    hawk.pages_copy(k, k, sv.int32([(n - 1, 520, 128), (3, n - 2, 100)]))
    assert (k[520] == 2.5).all() and (k[n - 2, :, :100] == 1.5).all() and (k[n - 2, :, 100:] == 0).all() and (k[519] == 0).all()


# ------------------------------------------------------------------------------------------ keep
def _trees(r, B, n, depth, first):
    path, accept = np.full((B, depth), -1, np.int64), []
    for b in range(B):
        count = int(r.randint(0, min(depth, n - first) + 1)) if n > first else 0
        path[b, :count] = np.sort(r.choice(np.arange(first, n), count, replace=False))
        accept.append(count)
    return path.tolist(), accept


@pytest.mark.parametrize("layout", ["hrd", "rhd", "kv"])
@pytest.mark.parametrize("page, n, first", [(16, 22, 1), (8, 64, 1), (1, 9, 2), (5, 130, 0), (64, 3, 1)])
def test_keep(page, n, first, layout):
    r = np.random.RandomState(n)
    B, H, D, layers = 3, 5, 64, 2
    S = 2 * B
    new = [n] * S
    new[4] = 0  # an idle stream
    kv = [n + int(x) for x in r.randint(0, 40, S)]
    st = sv.PageState(kv, page, serving.pages(max(kv), page), sum(serving.pages(x, page) for x in kv) + 2, seed=n)
    path, accept = _trees(r, B, n, 70, first)
    begin = np.concatenate([[2], 2 + np.cumsum(new)]).tolist()
    k, v = sv.pages_tensor(layers, st.n_pages, H, page, D, layout=layout, seed=n)
    want = [x.clone() for x in (k, v)]
    lens, moves = serving.keep(begin, kv, path, accept, first)
    for s, a, b in moves:
        for x in want:
            x[:, st.table[s][b // page], :, b % page] = x[:, st.table[s][a // page], :, a % page]
    table, kv_len, _ = st.cuda()
    status = _status()
    got = hawk.pages_keep(k, v, table, sv.int32(begin), kv_len, sv.int32(path), sv.int32(accept), first=first, dev_status=status)
    assert got.tolist() == lens and int(status) == 0 and torch.equal(k, want[0]) and torch.equal(v, want[1])
    # lengths alone, as for a chain
    assert hawk.pages_keep(None, None, None, sv.int32(begin), kv_len, None, sv.int32(accept), first=first).tolist() == lens


def test_keep_of_bad_paths_rows_and_pages():
    kv, page = [30, 30, 30, 30, 30, 30], 8
    st = sv.PageState(kv, page, 4, 30, seed=8)
    begin = sv.int32([0, 10, 20, 30, 40, 50, 60])
    k, v = sv.pages_tensor(0, 30, 2, page, 16)
    keep = k.clone()
    table, kv_len, _ = st.cuda()
    # descending, below `first`, past the rows, too many, negative, the same row twice
    path = sv.int32([[5, 4, -1], [0, 2, 3], [3, 9, 10], [2, 4, 6], [2, 4, 6], [4, 4, 5]])
    status = _status()
    got = hawk.pages_keep(k, v, table, begin, kv_len, path, sv.int32([2, 3, 3, 4, -1, 2]), dev_status=status)
    assert got.tolist() == kv and int(status) == binding.DEV_BAD_TREE and torch.equal(k, keep)
    status = _status()
    got = hawk.pages_keep(k, v, table, sv.int32([0, 10, 5, 30, 40, 50, 60]), sv.int32([30, 30, 8, 5, 33, 30]), sv.int32([[-1]] * 6),
                          sv.int32([0] * 6), dev_status=status)
    assert int(status) == binding.DEV_BAD_ROWS | binding.DEV_BAD_PREFIX and got.tolist() == [21, 30, 8, 5, 33, 21]
    table[0, 2] = 30
    status = _status()
    hawk.pages_keep(k, v, table, begin, kv_len, sv.int32([[3, 9, -1]] * 6), sv.int32([2, 0, 0, 0, 0, 0]), dev_status=status)
    assert int(status) == binding.DEV_BAD_PAGE
    with pytest.raises(binding.HawkError):
        hawk.pages_keep(k, v, table, begin, kv_len, path, sv.int32([0] * 6), out_len=kv_len)


# ------------------------------------------------------------------------------------------ graphs, streams, index checks
def test_captured_and_on_another_stream():
    st, r = _state(40, 16, 60)
    width = len(st.table[0])
    table, lens, refs = st.cuda()
    k, v = sv.pages_tensor(2, st.n_pages, 4, 16, 64)
    new, copies = torch.zeros_like(lens), torch.zeros((40, 3), dtype=torch.int32, device="cuda")
    out = dict(out_table=torch.zeros_like(table), out_len=torch.zeros_like(lens), out_refs=torch.zeros_like(refs), copies=copies)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hawk.pages_resize(table, lens, new, refs, 16, **out)
        hawk.pages_copy(k, v, copies)
        again = hawk.pages_compact(out["out_table"], out["out_len"], out["out_refs"], 16, 64)
        hawk.pages_copy(k, v, again)
    for seed in range(3):
        want_new = np.clip(np.array(st.lens) + np.random.RandomState(seed).randint(-30, 30, 40), 0, width * 16).tolist()
        new.copy_(sv.int32(want_new))
        graph.replay()
        t, n, c, cp, _ = serving.resize(st.table, st.lens, want_new, st.refs, 16)
        t, c, cp2, _ = serving.compact([[e if e is not None else 0 for e in row] for row in t], n, c, 16, 64)
        torch.cuda.synchronize()
        assert out["out_len"].tolist() == n and out["out_refs"].tolist() == c and sv.same_where_written(out["out_table"], t)
        assert [tuple(x) for x in again.tolist()] == cp2 and [tuple(x) for x in copies.tolist()] == cp


def test_no_index_leaves_its_array():
    lib = build.build_debug_variant()
    with binding.alternate_library(lib):
        for S, page in ((5, 16), (300, 3)):
            st, r = _state(S, page, 70 + S)
            new = [int(np.clip(n + r.choice([0, 9, -9, -n]), 0, len(st.table[0]) * page)) for n in st.lens]
            _same_resize(st, new, False)
            _compact(st, 300, False)
        test_keep(5, 130, 0, "hrd")


def test_refusals_with_tensors():
    st, _ = _state(4, 16, 80)
    table, lens, refs = st.cuda()
    with pytest.raises(TypeError, match="new_len: expected torch.int32"):
        hawk.pages_resize(table, lens, lens.long(), refs, 16)
    with pytest.raises(ValueError, match="kv_len: expected shape"):
        hawk.pages_resize(table, lens[:3], lens, refs, 16)
    with pytest.raises(ValueError, match="copies: expected shape"):
        hawk.pages_resize(table, lens, lens, refs, 16, copies=torch.zeros((4, 2), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="max_moves"):
        hawk.pages_compact(table, lens, refs, 16, -1)
    with pytest.raises(binding.HawkError):
        hawk.pages_resize(table, lens, lens, refs, 0)
    with pytest.raises(binding.HawkError):
        hawk.pages_compact(table, lens, refs, 16, 4, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    k, v = sv.pages_tensor(2, 5, 2, 16, 64)
    with pytest.raises(ValueError, match="v_pages"):
        hawk.pages_copy(k, v[0], sv.int32([[0, 1, 16]]))
    with pytest.raises(TypeError, match="k_pages"):
        hawk.pages_copy(k.float(), v, sv.int32([[0, 1, 16]]))


@pytest.mark.parametrize("S, S_out, width, n_pages", [(1, 32, 128, 4096), (32, 1, 128, 4095), (32, 32, 129, 4096), (33, 2, 4, 50), (2, 33, 4, 50),
                                                      (7, 9, 128, 4097), (3, 3, 5, 1), (0, 4, 3, 6), (5, 0, 3, 6)])
def test_fork_sizes_of_one_block(S, S_out, width, n_pages):
    """The sizes around which one block does it all: old streams with every page of the pool among them, some kept, some left."""
    page, r = 4, np.random.RandomState(S + width)
    lens = r.randint(0, width * page + 1, S)
    lens[:1] = width * page
    table = r.randint(0, n_pages, (S, width))
    refs = np.zeros(n_pages, np.int64)
    for s in range(S):
        np.add.at(refs, table[s, :serving.pages(int(lens[s]), page)], 1)
    parent, length = (r.randint(-1, S, S_out) if S else np.full(S_out, -1)), r.randint(0, width * page + 9, S_out)
    want = serving.fork(table.tolist(), lens.tolist(), parent.tolist(), refs.tolist(), page, length.tolist())
    args = [torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).cuda() for x in (table, lens, parent, refs, length)]
    for in_place in (False, True):
        out_refs, status = args[3] if in_place else torch.full_like(args[3], -5), _status()
        got_table, got_len = hawk.pages_fork(args[0], args[1], args[2], args[3], page, length=args[4], out_refs=out_refs, dev_status=status)
        assert int(status) == 0 and got_len.tolist() == want[1] and out_refs.tolist() == want[2]
        assert sv.same_where_written(got_table, want[0])


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S, spare", [(7, 60), (700, 4000)])
def test_streams_of_lengths_out_of_range_keep_their_entries(S, spare, in_place):
    """A stream with a sound length and a new one out of range stays as it is, entries included; one whose own length is out of range
    has none that could be told.  The others go on as if it were not asked."""
    page = 8
    st, r = _state(S, page, 90 + S, spare=spare)
    most = len(st.table[0]) * page
    new = [int(np.clip(n + r.randint(-20, 20), 0, most)) for n in st.lens]
    for s, bad in zip(range(0, S, 3), [-1, most + 1, -(1 << 31), (1 << 31) - 1] * S):
        new[s] = bad
    st.lens[1] = -3  # (its pages keep their counts)
    want_table, want_len, want_refs, want_copies, stayed = serving.resize(st.table, st.lens, new, st.refs, page)
    assert not stayed and want_len[::3] == st.lens[::3] and want_table[0][0] == st.table[0][0]
    table, lens, refs, copies, status = _resize(st, new, in_place)
    assert status == binding.DEV_BAD_PREFIX and lens.tolist() == want_len and refs.tolist() == want_refs
    assert [tuple(c) for c in copies.tolist()] == want_copies and sv.same_where_written(table, want_table)


@pytest.mark.parametrize("H, page, D", [(65536, 128, 128), (1, 16384, 65536), (2, 65531, 8192), (2, 65535, 8192)])
def test_copy_of_the_largest_pages(H, page, D):
    """Pages of 2^30 elements and a little less, in calls of few copies: as many blocks a page as a grid has."""
    k = torch.zeros((2, H, page, D), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 0] = 1.5
    k[0, H - 1, page - 2] = 2.5
    k[0, H // 2, page // 2, D // 2] = 3.5
    k[0, H - 1, page - 1] = 4.5
    hawk.pages_copy(k, k, sv.int32([(0, 1, page - 1)]))
    assert torch.equal(k[1, :, :page - 1], k[0, :, :page - 1]) and (k[1, :, page - 1] == 0).all()


@pytest.mark.parametrize("count", [0, -2])
@pytest.mark.parametrize("S, spare", [(5, 60), (700, 4000)])
def test_growing_into_a_page_without_a_count(S, spare, count):
    """A stream grows into a page that the counts say is free: flagged in every launch, also where the call hands that page to a stream."""
    page, width = 8, 16
    lens = [21] + [16] * (S - 1)
    n_pages = sum(serving.pages(n, page) for n in lens) + spare
    for seed, grown in ((0, 22), (1, 25), (2, 24)):
        st = sv.PageState(lens, page, width, n_pages, seed=seed)
        last = st.table[0][2]
        st.refs[last] = count
        new = [grown] + [16 + 8 * 2] * (S // 3) + [16] * (S - 1 - S // 3)
        want_table, want_len, want_refs, want_copies, stayed = serving.resize(st.table, st.lens, new, st.refs, page)
        for _ in range(4):
            table, got_len, refs, copies, status = _resize(st, new, False)
            assert status == binding.DEV_BAD_PAGE | (binding.DEV_NO_PAGES if stayed else 0)
            assert got_len.tolist() == want_len and refs.tolist() == want_refs and [tuple(c) for c in copies.tolist()] == want_copies
            assert sv.same_where_written(table, want_table)
    st = sv.PageState(lens, page, width, n_pages, seed=0)
    st.refs[st.table[0][2]] = count
    assert _resize(st, [21] + [16] * (S - 1), True)[4] == 0  # (who does not grow into it is not looked at)


def test_a_page_released_by_one_stream_while_another_that_names_it_grows():
    st = sv.PageState([21, 21], 8, 5, 30, share=2, seed=3, fresh=1.0)
    st.refs[st.table[0][2]] = 1  # two entries name it
    assert _resize(st, [0, 22], True)[4] == binding.DEV_BAD_PAGE


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("moves", [0, 5])
@pytest.mark.parametrize("S, n_pages", [(4, 16), (300, 4096)])
def test_compact_with_nothing_to_move_looks_at_lengths_and_ids(S, n_pages, moves, in_place):
    """A full pool: lengths and ids out of range are flagged as where pages move, and nothing changes."""
    st = sv.PageState([8 * (n_pages // S)] * S, 8, n_pages // S + 2, n_pages, seed=S)
    st.refs = [max(1, c) for c in st.refs]
    for what in ("length", "id", "both", "none"):
        table, lens, refs = st.cuda()
        want = 0
        if what in ("length", "both"):
            lens[S - 1], want = -1, want | binding.DEV_BAD_PREFIX
        if what in ("id", "both"):
            table[1, 2], want = n_pages, want | binding.DEV_BAD_PAGE
        out = {} if in_place else dict(out_table=torch.full_like(table, -9), out_refs=torch.zeros_like(refs))
        status, before = _status(), table.clone()
        copies = hawk.pages_compact(table, lens, refs, 8, moves, dev_status=status, **out)
        assert int(status) == want and (copies == torch.tensor([-1, -1, 0], device="cuda")).all()
        assert torch.equal(table, before) and out.get("out_refs", refs).tolist() == st.refs
        used = n_pages // S
        assert torch.equal(out.get("out_table", table)[:S - 1, :used], before[:S - 1, :used])


def test_tensors_without_elements():
    """Tables of no width, pages of no layers and paths of no columns have no address, and are not taken for missing."""
    none, zero = sv.int32(np.zeros((3, 0))), sv.int32([0, 0, 0])
    refs, status = sv.int32([0, 1, 0, 2, 0]), _status()
    for out in ({}, dict(out_table=sv.int32(np.zeros((3, 0))), out_len=sv.int32([5, 5, 5]), out_refs=sv.int32([9] * 5))):
        lens = zero.clone()
        copies = hawk.pages_resize(none, lens, sv.int32([0, 0, 1]), refs, 4, dev_status=status, **out)
        assert int(status) == binding.DEV_BAD_PREFIX and out.get("out_len", lens).tolist() == [0, 0, 0]
        assert out.get("out_refs", refs).tolist() == [0, 1, 0, 2, 0] and copies.tolist() == [[-1, -1, 0]] * 3
        status.zero_()
    for parents in ([2, -1], [0, 1, 2, 2]):
        to = torch.full_like(refs, 9)
        table, lens = hawk.pages_fork(none, zero, sv.int32(parents), refs, 4, out_refs=to, dev_status=status)
        assert table.shape == (len(parents), 0) and not lens.any() and torch.equal(to, refs)
    copies = hawk.pages_compact(none, zero, refs, 4, 2, dev_status=status)
    assert refs.tolist() == [2, 1, 0, 0, 0] and copies.tolist() == [[3, 0, 4], [-1, -1, 0]] and int(status) == 0
    # four streams of two sequences that brought three rows each; nothing was accepted, or so it should be
    begin, kv = sv.int32([0, 3, 6, 9, 12]), sv.int32([5, 6, 7, 8])
    k, v = sv.pages_tensor(2, 6, 2, 4, 8)
    table = sv.int32([[0, 1], [2, 3], [4, 5], [0, 2]])
    keep = k.clone()
    got = hawk.pages_keep(k, v, table, begin, kv, sv.int32(np.zeros((2, 0))), sv.int32([0, 0]), dev_status=status)
    assert got.tolist() == [3, 4, 5, 6] and int(status) == 0
    got = hawk.pages_keep(k, v, table, begin, kv, sv.int32(np.zeros((2, 0))), sv.int32([1, 0]), dev_status=status)
    assert got.tolist() == [5, 4, 7, 6] and int(status) == binding.DEV_BAD_TREE and torch.equal(k, keep)
    status.zero_()
    got = hawk.pages_keep(k[:0], v[:0], table, begin, kv, sv.int32([[2], [1]]), sv.int32([1, 0]), dev_status=status)
    assert got.tolist() == [4, 4, 6, 6] and int(status) == 0


# ------------------------------------------------------------------------------------------ what goes wrong in states of many pages
def _large(seed, spare=3000, share=2):
    """700 streams over more pages than one block takes."""
    return _state(700, 8, seed, share=share, spare=spare)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("left", [0, 1, 77, 150, 333])
def test_pages_run_out_in_the_middle_of_a_large_batch(left, in_place):
    """All but `left` free pages, spread over the pool, are held by the caller: the first stream that finds too few lies somewhere in the
    batch, and the last free page somewhere in a block's share."""
    for seed in (1, 2):
        st, r = _large(100 + seed)
        free = [p for p, c in enumerate(st.refs) if c == 0]
        for p in r.permutation(free)[left:]:
            st.refs[p] = 1
        most = len(st.table[0]) * 8
        new = [int(np.clip(n + r.choice([0, 3, 9, 40, -9, -n]), 0, most)) for n in st.lens]
        want = serving.resize(st.table, st.lens, new, st.refs, 8)
        assert st.n_pages > 2048 and want[4]
        _same_resize(st, new, in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_page_ids_out_of_range_in_a_large_batch(in_place):
    """Ids that are none, in entries that are released and in those that streams grow into: flagged by every block, counted by none."""
    st, r = _large(110)
    n, page = st.n_pages, 8
    new, bad, expect = list(st.lens), [-1, n, 1 << 30, -(1 << 31)], list(st.refs)
    cut = [s for s in range(700) if st.lens[s] > 16][::9]
    grow = [s for s in range(700) if st.lens[s] % page and s not in cut][::7]
    table = [list(row) for row in st.table]
    for i, s in enumerate(cut):  # releases its last two entries, of which one is none
        new[s] = (serving.pages(st.lens[s], page) - 2) * page
        at = serving.pages(st.lens[s], page) - 1 - i % 2
        table[s][at] = bad[i % 4]
        expect[table[s][serving.pages(st.lens[s], page) - 2 + i % 2]] -= 1
    for i, s in enumerate(grow):  # within its last page, which is none
        if st.lens[s] % page == page - 1:
            continue
        new[s] = st.lens[s] + 1 if (st.lens[s] + 1) % page else st.lens[s]
        if new[s] > st.lens[s]:
            table[s][st.lens[s] // page] = bad[i % 4]
    dev_table, lens, refs = sv.int32(table), sv.int32(st.lens), sv.int32(st.refs)
    status = _status()
    out = {} if in_place else dict(out_table=torch.full_like(dev_table, -9), out_len=torch.zeros_like(lens), out_refs=torch.zeros_like(refs))
    copies = hawk.pages_resize(dev_table, lens, sv.int32(new), refs, page, dev_status=status, **out)
    assert int(status) == binding.DEV_BAD_PAGE and out.get("out_len", lens).tolist() == new
    assert out.get("out_refs", refs).tolist() == expect and (copies[:, 0] == -1).all()
    got = out.get("out_table", dev_table).tolist()
    assert all(got[s][:serving.pages(new[s], page)] == table[s][:serving.pages(new[s], page)] for s in range(700))


@pytest.mark.parametrize("in_place", [True, False])
def test_compact_of_a_large_table_that_names_free_pages(in_place):
    """As for a small one: the entry stays and is flagged, whatever the workspace held before."""
    st, _ = _large(120, share=1)
    free = [p for p, c in enumerate(st.refs) if c == 0][::-1][:6]
    where = [s for s in range(700) if st.lens[s] > 0][::130][:6]
    table, refs = [list(row) for row in st.table], list(st.refs)
    for s, p in zip(where, free):
        refs[table[s][0]], table[s][0] = 0, p
    for fill in (0, 1, 255):
        for moves in (3, 900, st.n_pages):
            want_table, want_refs, want_copies, want_top = serving.compact(table, st.lens, refs, 8, moves)
            moved = [a for a, _, _ in want_copies if a >= 0]
            ws = torch.full((hawk.pages_compact_workspace_bytes(st.n_pages, moves),), fill, dtype=torch.uint8, device="cuda")
            dev_table, dev_refs, lens, status, top = sv.int32(table), sv.int32(refs), sv.int32(st.lens), _status(), _status()
            out = {} if in_place else dict(out_table=torch.full_like(dev_table, -9), out_refs=torch.zeros_like(dev_refs))
            copies = hawk.pages_compact(dev_table, lens, dev_refs, 8, moves, workspace=ws, top=top, dev_status=status, **out)
            assert int(status) == (binding.DEV_BAD_PAGE if max(free) >= min(moved) else 0)
            assert sv.same_where_written(out.get("out_table", dev_table), want_table)
            assert out.get("out_refs", dev_refs).tolist() == want_refs and [tuple(c) for c in copies.tolist()] == want_copies
            assert int(top) == want_top


def test_no_index_leaves_its_array_in_a_large_batch():
    lib = build.build_debug_variant()
    with binding.alternate_library(lib):
        test_pages_run_out_in_the_middle_of_a_large_batch(333, False)
        test_page_ids_out_of_range_in_a_large_batch(False)
        test_compact_of_a_large_table_that_names_free_pages(False)
