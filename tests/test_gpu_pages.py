"""hook_pages_fork, hook_pages_append and hook_pages_compact against their definitions, and the contents of the caches through
many steps of them (needs an MI355X)."""
import random

import pytest
import torch

from oracle import generation as G
from paper_2603_06588_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
JUNK = -123456789      # in table entries that no call may read or write


def ints(x, shape=None):
    t = torch.tensor(x, dtype=torch.int32, device=DEV)
    return t if shape is None else t.view(shape)


class Pool:
    """A consistent random state: rows that share prefixes of each other's pages, pages held by somebody else, free pages."""

    def __init__(self, seed, S, mb, most, spare, share=0.5, held_elsewhere=0.2):
        r = random.Random(seed)
        pages = iter(range(10 ** 9))
        self.rows, self.lens = [], []
        for i in range(S):
            n = r.choice([0, 1, 15, 16, 17, r.randint(0, most), r.randint(0, most)])
            n = min(n, most, mb * 16)
            have = -(-n // 16)
            row = []
            if i and r.random() < share:
                j = r.randrange(i)
                if r.random() < 0.5:
                    n = min(self.lens[j], n) if r.random() < 0.5 else self.lens[j]      # all of it, or a prefix
                    have = -(-n // 16)
                row = self.rows[j][:min(have, self.lens[j] // 16 if have > len(self.rows[j]) else have)]
            row = row + [next(pages) for _ in range(have - len(row))]
            self.rows.append(row)
            self.lens.append(n)
        used = next(pages)
        elsewhere = int(used * held_elsewhere)
        nb = used + elsewhere + spare + 1
        ids = list(range(nb))
        r.shuffle(ids)
        self.rows = [[ids[p] for p in row] for row in self.rows]
        self.refs = [0] * nb
        for row in self.rows:
            for p in row:
                self.refs[p] += 1
        for p in ids[used:used + elsewhere]:
            self.refs[p] += 1
        for p in ids[:used]:
            if r.random() < 0.1:
                self.refs[p] += 1
        self.S, self.mb, self.nb = S, mb, nb

    def table(self):
        return [row + [JUNK] * (self.mb - len(row)) for row in self.rows]


def check_table(got, rows, before=None):
    """The rows' pages, and the entries behind them as they were."""
    got = got.cpu().tolist()
    for i, row in enumerate(rows):
        assert got[i][:len(row)] == row, (i, got[i][:len(row)], row)
        rest = [JUNK] * (len(got[i]) - len(row)) if before is None else before[i][len(row):]
        assert got[i][len(row):] == rest, i


STATES = [(1, 1, 16, 3), (1, 4, 60, 9), (3, 8, 100, 20), (9, 40, 500, 60), (64, 30, 400, 200), (65, 1100, 17000, 50), (300, 20, 300, 900), (7, 2100, 30000, 2500), (900, 12, 150, 400), (1500, 6, 80, 300), (3, 4500, 71000, 10)]


@pytest.mark.parametrize("S,mb,most,spare", STATES)
@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("apart", [False, True])
def test_fork(S, mb, most, spare, cut, apart):
    p = Pool(S + mb, S, mb, most, spare)
    r = random.Random(S)
    for N in {1, S, 2 * S + 3}:
        src = [r.choice([-1, r.randrange(S), r.randrange(S)]) for _ in range(N)]
        keep = [r.choice([0, -5, 10 ** 9, r.randint(0, most)]) for _ in range(N)] if cut else None
        table, lens, refs = ints(p.table(), (S, mb)), ints(p.lens), ints(p.refs)
        out, lens_out = torch.full((N, mb), JUNK, dtype=torch.int32, device=DEV), torch.full((N,), 77, dtype=torch.int32, device=DEV)
        status = ints([64])
        refs_out = torch.full_like(refs, 99) if apart else None
        binding.hook_pages_fork(ints(src), table, lens, refs, out, lens_out, status, src_lens=None if keep is None else ints(keep), ref_counts_out=refs_out)
        rows, L, counts, bits = G.fork(src, p.table(), p.lens, p.refs, keep)
        check_table(out, rows)
        assert lens_out.tolist() == L and (refs_out if apart else refs).tolist() == counts and int(status) == 64 | bits
        assert not apart or refs.tolist() == p.refs
        check_table(table, p.rows)


def test_fork_of_bad_input_is_safe():
    table = [[0, 99, JUNK], [1, -3, 2], [2, 0, 1]]
    lens, refs, src, keep = [32, 48, 100], [2, 2, 2], [2, 7, -2, 1, 0], [1000] * 5
    out, lens_out, status, counts = ints([[JUNK] * 3] * 5), ints([0] * 5), ints([0]), ints(refs)
    binding.hook_pages_fork(ints(src), ints(table), ints(lens), counts, out, lens_out, status, src_lens=ints(keep))
    rows, L, want, bits = G.fork(src, table, lens, refs, keep)
    assert bits == G.BAD_ROW | G.BAD_LENGTH | G.BAD_PAGE
    check_table(out, rows)
    assert lens_out.tolist() == L and counts.tolist() == want and int(status) == bits
    # a negative length
    status.zero_()
    binding.hook_pages_fork(ints([0]), ints([[1]]), ints([-4]), counts, out[:1, :1].contiguous(), lens_out[:1], status)
    assert int(lens_out[0]) == 0 and int(status) == G.BAD_LENGTH


@pytest.mark.parametrize("S", [40, 1300])
def test_fork_that_only_reorders(S):
    """Every row goes on in another place: no count changes, and a row named twice counts once more."""
    p = Pool(S, S, 10, 150, 50)
    order = list(range(S))
    random.Random(S).shuffle(order)
    for src in (order, list(range(S)), order[:-1] + [order[0]]):
        refs, out, lens, status = ints(p.refs), torch.full((S, 10), JUNK, dtype=torch.int32, device=DEV), ints([0] * S), ints([0])
        binding.hook_pages_fork(ints(src), ints(p.table()), ints(p.lens), refs, out, lens, status)
        rows, L, counts, bits = G.fork(src, p.table(), p.lens, p.refs)
        check_table(out, rows)
        assert lens.tolist() == L and refs.tolist() == counts and int(status) == bits == 0


def test_fork_from_and_to_no_rows():
    refs, status = ints([1, 0, 1]), ints([0])
    none, empty = torch.empty((0, 2), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    binding.hook_pages_fork(empty, ints([[2, 0]]), ints([20]), refs, none, empty, status)      # everything is freed
    assert refs.tolist() == [0, 0, 0] and int(status) == 0
    out, lens = ints([[5, 5]]), ints([3])
    binding.hook_pages_fork(ints([-1]), none, empty, refs, out, lens, status)
    assert lens.tolist() == [0] and out.tolist() == [[5, 5]] and refs.tolist() == [0, 0, 0]


def new_caches(nb, heads, d, dtype, count, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-2 ** 15, 2 ** 15, (count, nb, heads, 16, d * (2 if dtype == torch.float32 else 1)), generator=g).to(torch.int16).to(DEV)


def run_append(p, cu, caches, apart, status, as_list=False):
    table, lens, refs = ints(p.table(), (p.S, p.mb)), ints(p.lens), ints(p.refs)
    kw = {}
    if apart:
        kw = {"block_table_out": torch.full_like(table, JUNK), "seq_lens_out": torch.full_like(lens, 5), "ref_counts_out": torch.full_like(refs, 5)}
    binding.hook_pages_append(ints(cu), table, lens, refs, list(caches) if as_list else caches, status, **kw)
    if apart:
        check_table(table, p.rows)
        assert lens.tolist() == p.lens and refs.tolist() == p.refs
        return kw["block_table_out"], kw["seq_lens_out"], kw["ref_counts_out"]
    return table, lens, refs


@pytest.mark.parametrize("S,mb,most,spare", STATES)
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("new", [1, 40])
def test_append(S, mb, most, spare, apart, new):
    if mb * 16 <= new:
        pytest.skip("no room for so many tokens in a row")
    r = random.Random(S + new)
    # enough room in the table and in the cache
    p = Pool(S * 3 + mb, S, mb, min(most, mb * 16 - new), S * (new // 16 + 2), share=0.7)
    cu = [0]
    for _ in range(S):
        cu.append(cu[-1] + r.choice([0, 1, r.randint(0, new)]))
    caches = new_caches(p.nb, 2, 32, torch.bfloat16, 3)
    before, status = caches.clone(), ints([0])
    table, lens, refs = run_append(p, cu, caches, apart, status, as_list=S % 2 == 0)
    rows, L, counts, copies, bits = G.append(cu, p.table(), p.lens, p.refs)
    assert bits == 0
    check_table(table, rows)
    assert lens.tolist() == L and refs.tolist() == counts and int(status) == 0
    for a, b, n in copies:
        before[:, b, :, :n] = before[:, a, :, :n]
    assert torch.equal(caches, before)


@pytest.mark.parametrize("S", [2, 70, 513])
def test_append_to_pages_with_many_holders(S):
    """Every row shares one page; all but the last holder copy it, unless somebody else holds it too."""
    for more in (0, 1):
        nb = S + 3
        p = Pool.__new__(Pool)
        p.S, p.mb, p.nb, p.rows, p.lens, p.refs = S, 2, nb, [[nb - 1]] * S, [5] * S, [0] * (nb - 1) + [S + more]
        cu = list(range(S + 1))
        caches, status = new_caches(nb, 1, 16, torch.bfloat16, 2), ints([0])
        before = caches.clone()
        table, lens, refs = run_append(p, cu, caches, False, status)
        rows, L, counts, copies, bits = G.append(cu, p.table(), p.lens, p.refs)
        assert len(copies) == S - 1 + more and bits == 0
        check_table(table, rows)
        assert lens.tolist() == L and refs.tolist() == counts and int(status) == 0
        for a, b, n in copies:
            before[:, b, :, :n] = before[:, a, :, :n]
        assert torch.equal(caches, before)


@pytest.mark.parametrize("why", ["pages", "copy", "row"])
@pytest.mark.parametrize("apart", [False, True])
def test_append_is_all_or_nothing(why, apart):
    p = Pool.__new__(Pool)
    p.S, p.mb, p.nb = 3, 3, 6
    p.rows, p.lens, p.refs = [[0, 1], [0, 1], [2]], [20, 20, 16], [2, 2, 1, 0, 0, 1]
    cu = {"pages": [0, 1, 1, 33], "copy": [0, 1, 2, 34], "row": [0, 0, 29, 29]}[why]
    if why == "pages":
        p.refs[3] = 7
    caches, status = new_caches(6, 1, 16, torch.bfloat16, 1), ints([0])
    if why == "copy":
        p.refs[4] = 1
    before = caches.clone()
    rows, L, counts, copies, bits = G.append(cu, p.table(), p.lens, p.refs)
    table, lens, refs = run_append(p, cu, caches, apart, status)
    assert bits == G.FULL and int(status) == G.FULL
    check_table(table, p.rows)
    assert lens.tolist() == p.lens and refs.tolist() == p.refs and torch.equal(caches, before)


def test_append_of_bad_input_is_safe():
    table, lens, refs = [[0, 77], [1, 0], [2, 0]], [20, -9, 5], [1, 0, 1, 0]
    cu = [0, 1, 2, 1]
    caches, status = new_caches(4, 1, 16, torch.bfloat16, 1), ints([0])
    before = caches.clone()
    t, L, counts = ints(table), ints(lens), ints(refs)
    binding.hook_pages_append(ints(cu), t, L, counts, caches, status)
    rows, want_l, want, copies, bits = G.append(cu, table, lens, refs)
    assert bits == G.BAD_LENGTH | G.BAD_PAGE and int(status) == bits and copies == []
    check_table(t, rows, table)
    assert L.tolist() == want_l and counts.tolist() == want and torch.equal(caches, before)


def test_bookkeeping_alone():
    p = Pool(5, 6, 10, 100, 30)
    cu, status = list(range(7)), ints([0])
    table, lens, refs = run_append(p, cu, [], False, status)
    rows, L, counts, _, bits = G.append(cu, p.table(), p.lens, p.refs)
    check_table(table, rows)
    assert lens.tolist() == L and refs.tolist() == counts and bits == 0
    t, r, m, n = ints(p.table()), ints(p.refs), ints([9] * p.nb), ints([9])
    binding.hook_pages_compact(t, ints(p.lens), r, [], m, n, status)
    rows, counts, page_map, live, _, _ = G.compact(p.table(), p.lens, p.refs)
    check_table(t, rows)
    assert r.tolist() == counts and m.tolist() == page_map and int(n) == live and int(status) == 0


@pytest.mark.parametrize("S,mb,most,spare", STATES + [(2, 4, 30, 5000), (3, 3000, 40000, 0)])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("heads,d,dtype", [(2, 32, torch.bfloat16), (3, 8, torch.float32)])
def test_compact(S, mb, most, spare, apart, heads, d, dtype):
    p = Pool(S + 7 * mb, S, mb, most, spare)
    caches = new_caches(p.nb, heads, d, dtype, 2)
    before, status = caches.clone(), ints([0])
    table, refs = ints(p.table(), (S, mb)), ints(p.refs)
    page_map, live = ints([55] * p.nb), ints([0])
    kw = {"block_table_out": torch.full_like(table, JUNK), "ref_counts_out": torch.full_like(refs, 5)} if apart else {}
    binding.hook_pages_compact(table, ints(p.lens), refs, caches, page_map, live, status, **kw)
    rows, counts, want_map, n, moves, bits = G.compact(p.table(), p.lens, p.refs)
    check_table(kw.get("block_table_out", table), rows)
    assert kw.get("ref_counts_out", refs).tolist() == counts and page_map.tolist() == want_map and int(live) == n and int(status) == bits == 0
    for a, b in moves:
        before[:, b] = before[:, a]
    assert torch.equal(caches, before)
    if apart:
        check_table(table, p.rows)
        assert refs.tolist() == p.refs


@pytest.mark.parametrize("nb", [1, 2047, 2048, 2049, 6000])
@pytest.mark.parametrize("full", [0.0, 0.3, 1.0])
def test_compact_at_chunk_borders(nb, full):
    r = random.Random(nb)
    refs = [int(r.random() < full) * r.randint(1, 3) for _ in range(nb)]
    table = [[p for p in range(nb) if refs[p]] or [JUNK]]
    lens = [16 * sum(x > 0 for x in refs)]
    caches, status = new_caches(nb, 1, 8, torch.bfloat16, 1), ints([0])
    before = caches.clone()
    t, c, page_map, live = ints(table), ints(refs), ints([0] * nb), ints([0])
    binding.hook_pages_compact(t, ints(lens), c, caches, page_map, live, status)
    rows, counts, want_map, n, moves, bits = G.compact(table, lens, refs)
    check_table(t, rows, table)
    assert c.tolist() == counts and page_map.tolist() == want_map and int(live) == n and int(status) == 0
    for a, b in moves:
        before[:, b] = before[:, a]
    assert torch.equal(caches, before)


def test_compact_of_bad_input_is_safe():
    table, lens, refs = [[3, 9, 1], [2, 0, 5]], [48, 99], [0, 0, 1, 1, 0, 2]
    t, c, page_map, live, status = ints(table), ints(refs), ints([0] * 6), ints([0]), ints([0])
    caches = new_caches(6, 1, 8, torch.bfloat16, 1)
    binding.hook_pages_compact(t, ints(lens), c, caches, page_map, live, status)
    rows, counts, want_map, n, _, bits = G.compact(table, lens, refs)
    assert bits == G.BAD_PAGE | G.BAD_LENGTH and int(status) == bits
    check_table(t, rows, table)
    assert c.tolist() == counts and page_map.tolist() == want_map and int(live) == n


def test_pages_at_far_offsets():
    """Pages of 4 MiB: the last ones begin behind 2^31 and 2^32 bytes."""
    heads, row = 64, 4096
    nb = 1040
    cache = torch.zeros((nb, heads, 16, row), dtype=torch.uint8, device=DEV)
    cache[nb - 1, :, :, :] = 7
    cache[nb - 1, heads - 1, 4, row - 1] = 9
    refs = [0] * nb
    refs[nb - 1] = 2
    status = ints([0])
    table, lens, counts = ints([[nb - 1], [nb - 1]]), ints([5, 5]), ints(refs)
    binding.hook_pages_append(ints([0, 1, 1]), table, lens, counts, [cache], status)
    assert table.tolist() == [[0], [nb - 1]] and int(cache[0, heads - 1, 4, row - 1]) == 9 and int(cache[0, :, 5:].max()) == 0 and int(cache[0, :, :5].min()) == 7
    page_map, live = ints([0] * nb), ints([0])
    binding.hook_pages_compact(table, lens, counts, [cache], page_map, live, status)
    assert table.tolist() == [[0], [1]] and torch.equal(cache[1], cache[nb - 1]) and int(status) == 0


def test_captured_graph_of_a_step():
    """fork, append and compact in a graph, replayed on fresh states: each replay gives what the calls give."""
    S, mb = 12, 20
    p = Pool(11, S, mb, 200, 60)
    r = random.Random(2)
    caches = new_caches(p.nb, 2, 16, torch.bfloat16, 2)
    start = [ints(p.table()), ints(p.lens), ints(p.refs), caches.clone()]
    src = ints([r.randrange(S) for _ in range(S)])
    cu = ints(list(range(S + 1)))

    def state():
        return [t.clone() for t in start] + [torch.full((S, mb), JUNK, dtype=torch.int32, device=DEV), ints([0] * S), ints([0] * p.nb), ints([0]), ints([0])]

    workspace = torch.empty(binding.pages_workspace_bytes(S, p.nb), dtype=torch.uint8, device=DEV)

    def step(s):
        table, lens, refs, caches, out, lens_out, page_map, live, status = s
        binding.hook_pages_fork(src, table, lens, refs, out, lens_out, status)
        binding.hook_pages_append(cu, out, lens_out, refs, caches, status, workspace=workspace)
        binding.hook_pages_compact(out, lens_out, refs, caches, page_map, live, status, workspace=workspace)

    eager, kept = state(), state()
    step(eager)
    step(kept)      # (warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kept)
    for _ in range(3):
        for t, fresh in zip(kept, state()):
            t.copy_(fresh)
        workspace.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager))


@pytest.mark.parametrize("which", [(0,), (1,), (2,), (0, 1), (1, 2), (0, 2)])
def test_append_with_some_outputs_in_place(which):
    """Table, lengths and counts may each be in place or not."""
    p = Pool(21, 20, 12, 120, 40, share=0.8)
    cu, status = list(range(21)), ints([0])
    caches = new_caches(p.nb, 1, 16, torch.bfloat16, 2)
    before = caches.clone()
    ins = [ints(p.table()), ints(p.lens), ints(p.refs)]
    outs = [t if i in which else torch.full_like(t, JUNK) for i, t in enumerate(ins)]
    binding.hook_pages_append(ints(cu), *ins, caches, status, block_table_out=outs[0], seq_lens_out=outs[1], ref_counts_out=outs[2])
    rows, L, counts, copies, bits = G.append(cu, p.table(), p.lens, p.refs)
    check_table(outs[0], rows)
    assert outs[1].tolist() == L and outs[2].tolist() == counts and int(status) == bits == 0 and len(copies) > 3
    for a, b, n in copies:
        before[:, b, :, :n] = before[:, a, :, :n]
    assert torch.equal(caches, before)


def test_many_caches_and_another_stream():
    """More caches than the short argument list holds, on a stream that is not the current one, with the call's own scratch."""
    p = Pool(31, 30, 12, 150, 60, share=0.8)
    caches = list(new_caches(p.nb, 1, 16, torch.bfloat16, 40))
    cu, status = ints(list(range(31))), ints([0])
    t, L, c, page_map, live = ints(p.table()), ints(p.lens), ints(p.refs), ints([0] * p.nb), ints([0])
    want = [x.clone() for x in caches]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.hook_pages_append(cu, t, L, c, caches, status, stream=side)
    binding.hook_pages_compact(t, L, c, caches, page_map, live, status, stream=side)
    side.synchronize()
    rows, lens, counts, copies, bits = G.append(list(range(31)), p.table(), p.lens, p.refs)
    table = [r + [JUNK] * (12 - len(r)) for r in rows]
    rows, counts, want_map, n, moves, _ = G.compact(table, lens, counts)
    check_table(t, rows)
    assert L.tolist() == lens and c.tolist() == counts and page_map.tolist() == want_map and int(live) == n and int(status) == 0
    for x in want:
        for a, b, k in copies:
            x[b, :, :k] = x[a, :, :k]
        for a, b in moves:
            x[b] = x[a]
    assert all(torch.equal(x, y) for x, y in zip(caches, want))


def test_more_pages_than_segments():
    """Over 256 chunks of 2048 pages: several chunks to a segment, free and live pages far apart."""
    nb = 2048 * 600 + 77
    g = torch.Generator().manual_seed(1)
    refs = torch.ones(nb, dtype=torch.int32)
    free = torch.randperm(nb, generator=g)[:5000]
    refs[free] = 0
    refs[2048 * 100:2048 * 300] = 0            # whole chunks without a live page
    table, lens = [[nb - 1] + [0] * 400, [2048 * 350 + 5] + [0] * 400], [16, 5]
    refs[nb - 1], refs[2048 * 350 + 5] = 1, 2
    t, L, c, status = ints(table), ints(lens), refs.to(DEV), ints([0])
    binding.hook_pages_append(ints([0, 6000, 6001]), t, L, c, [], status)
    order = (refs == 0).nonzero()[:, 0].tolist()
    want = [[nb - 1] + order[:375], [order[375]]]
    check_table(t, want, table)
    refs[order[:376]] = 1
    refs[2048 * 350 + 5] = 1
    assert L.tolist() == [6016, 6] and torch.equal(c.cpu(), refs) and int(status) == 0
    page_map, live = torch.empty(nb, dtype=torch.int32, device=DEV), ints([0])
    binding.hook_pages_compact(t, L, c, [], page_map, live, status)
    alive = refs > 0
    n = int(alive.sum())
    at = torch.arange(nb)
    movers, holes = at[alive & (at >= n)], at[~alive & (at < n)]
    want_map = torch.where(alive, at, -1)
    want_map[movers] = holes
    assert int(live) == n and torch.equal(page_map.cpu().long(), want_map) and int(status) == 0
    check_table(t, [[int(want_map[p]) for p in row] for row in want], table)
    assert torch.equal(c.cpu() > 0, at < n)


def test_refusals_of_the_binding():
    i, t = ints([0]), ints([[0, 0]])
    c = torch.zeros((1, 1, 16, 8), dtype=torch.bfloat16, device=DEV)
    fork = dict(src_rows=i, block_table=t, seq_lens=i, ref_counts=ints([0]), block_table_out=t.clone(), seq_lens_out=ints([0]), status=ints([0]))
    for bad in (dict(src_rows=i.long()), dict(block_table_out=t.view(2, 1).clone()), dict(block_table_out=t), dict(seq_lens_out=i), dict(block_table_out=ints([[0]])), dict(status=ints([0, 0])), dict(src_lens=ints([1, 2])),
                dict(block_table=t.cpu()), dict(ref_counts_out=ints([0, 0]))):
        with pytest.raises(binding.HookError):
            binding.hook_pages_fork(**{**fork, **bad})
    app = dict(cu_q_lens=ints([0, 0]), block_table=t, seq_lens=i, ref_counts=ints([0]), caches=[c], status=ints([0]))
    for bad in (dict(cu_q_lens=i), dict(caches=[c, c.float()]), dict(caches=[c[:, :, :8]]), dict(caches=[c.cpu()]), dict(caches=[torch.zeros((2, 1, 16, 8), device=DEV)]),
                dict(caches=[c.transpose(2, 3)]), dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), dict(caches=[torch.zeros((1, 1, 16, 4), dtype=torch.bfloat16, device=DEV)])):
        with pytest.raises(binding.HookError):
            binding.hook_pages_append(**{**app, **bad})
    com = dict(block_table=t, seq_lens=i, ref_counts=ints([0]), caches=[c], page_map=ints([0]), num_live=ints([0]), status=ints([0]))
    for bad in (dict(page_map=ints([0, 0])), dict(num_live=ints([0, 0])), dict(block_table_out=ints([[0]]))):
        with pytest.raises(binding.HookError):
            binding.hook_pages_compact(**{**com, **bad})


def test_scratch_of_a_call_on_another_stream_is_that_streams(monkeypatch):
    """The call's own scratch is taken while the call's stream is the current one."""
    p = Pool(41, 9, 12, 150, 60, share=0.8)
    side, taken, empty = torch.cuda.Stream(), [], torch.empty
    caches, status = new_caches(p.nb, 1, 16, torch.bfloat16, 2), ints([0])
    t, L, c, page_map, live, cu = ints(p.table()), ints(p.lens), ints(p.refs), ints([0] * p.nb), ints([0]), ints(list(range(10)))
    side.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(binding.torch, "empty", lambda *a, **kw: taken.append(torch.cuda.current_stream()) or empty(*a, **kw))
    binding.hook_pages_append(cu, t, L, c, caches, status, stream=side)
    binding.hook_pages_compact(t, L, c, caches, page_map, live, status, stream=side)
    monkeypatch.undo()
    side.synchronize()
    assert taken == [side, side] and torch.cuda.current_stream() != side
    rows, lens, counts, _, _ = G.append(list(range(10)), p.table(), p.lens, p.refs)
    assert L.tolist() == lens and int(live) == sum(n > 0 for n in counts) and int(status) == 0


@pytest.mark.parametrize("missing", ["src_rows", "block_table_out", "seq_lens_out"])
def test_fork_without_its_tensors_is_refused(missing):
    refs, table = ints([1, 1]), ints([[0], [1]])
    args = dict(src_rows=ints([0, 1]), block_table=table, seq_lens=ints([9, 9]), ref_counts=refs, block_table_out=torch.empty_like(table),
                seq_lens_out=ints([0, 0]), status=ints([0]))
    with pytest.raises(binding.HookError) as e:
        binding.hook_pages_fork(**{**args, missing: None})
    assert e.value.status == 1 and refs.tolist() == [1, 1]


@pytest.mark.parametrize("mb", [1, 5000])
def test_fork_of_no_rows_into_no_rows_hands_the_counts_on(mb):
    none, empty = torch.empty((0, mb), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    refs, counts, status = ints([3, 0, 1] * 100), ints([99] * 300), ints([0])
    binding.hook_pages_fork(empty, none, empty, refs, none.clone(), empty.clone(), status, ref_counts_out=counts)
    assert counts.tolist() == refs.tolist() == [3, 0, 1] * 100 and int(status) == 0
    binding.hook_pages_fork(empty, none, empty, refs, none.clone(), empty.clone(), status)
    assert refs.tolist() == [3, 0, 1] * 100 and int(status) == 0


def test_append_looks_at_the_last_page_alone():
    table, lens, refs, cu = [[99, 0, 7], [99, 7, 7], [99, 7, 7]], [20, 9, 16], [1, 0, 0], [0, 1, 1, 2]
    t, L, c, status = ints(table), ints(lens), ints(refs), ints([0])
    binding.hook_pages_append(ints(cu), t, L, c, [], status)
    rows, want_l, want, _, bits = G.append(cu, table, lens, refs)
    check_table(t, rows, table)
    assert L.tolist() == want_l and c.tolist() == want and int(status) == bits == 0
