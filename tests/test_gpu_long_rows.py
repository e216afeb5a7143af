"""Rows of more pages than one turn of a fork's counting workgroups takes (4096 columns), in tables that no other test fills that far: fork, append and
compact against their definitions (needs an MI355X)."""
import random

import pytest
import torch

from oracle import generation as G
from paper_2603_06588_amd import binding
from test_gpu_pages import DEV, JUNK, ints, new_caches

pytestmark = pytest.mark.gpu
TURN = 4096      # columns


class Table:
    """Rows by their lengths: row i takes the first `shared` pages of row `of` (both from `share[i]`) and new ones for the rest; every tenth page is also
    held by somebody else."""

    def __init__(self, lens, share, mb, spare, seed):
        r = random.Random(seed)
        self.lens, self.mb, self.S = list(lens), mb, len(lens)
        rows, used = [], 0
        for i, n in enumerate(lens):
            of, shared = share.get(i, (0, 0))
            row = rows[of][:shared] if shared else []
            row = row[:-(-n // 16)]
            row = row + list(range(used, used + -(-n // 16) - len(row)))
            used = max(used, (row or [0])[-1] + 1)
            rows.append(row)
        self.nb = used + spare
        ids = list(range(self.nb))
        r.shuffle(ids)
        self.rows, self.refs = [[ids[p] for p in row] for row in rows], [0] * self.nb
        for row in self.rows:
            for p in row:
                self.refs[p] += 1
        for p in ids[:used:10]:
            self.refs[p] += 1
        assert max(len(row) for row in self.rows) > TURN

    def tensor(self):
        return as_tensor(self.rows, self.mb)

    def short(self):
        """The rows as the definitions take them: no entries behind a row's pages but in the first row, which says how wide the table is."""
        return [self.rows[0] + [JUNK] * (self.mb - len(self.rows[0]))] + self.rows[1:]


def as_tensor(rows, mb):
    t = torch.full((len(rows), mb), JUNK, dtype=torch.int32)
    for i, row in enumerate(rows):
        t[i, :len(row)] = torch.tensor(row, dtype=torch.int32)
    return t


def check_fork(t, src, keep):
    for apart in (False, True):
        table, refs, status = t.tensor().to(DEV), ints(t.refs), ints([0])
        out, lens_out = torch.full((len(src), t.mb), JUNK, dtype=torch.int32, device=DEV), ints([77] * len(src))
        counts = torch.full_like(refs, 99) if apart else None
        binding.hook_pages_fork(ints(src), table, ints(t.lens), refs, out, lens_out, status, src_lens=None if keep is None else ints(keep), ref_counts_out=counts)
        rows, L, want, bits = G.fork(src, t.short(), t.lens, t.refs, keep)
        assert bits == 0 and int(status) == 0 and lens_out.tolist() == L
        assert torch.equal(out.cpu(), as_tensor(rows, t.mb)) and torch.equal(table.cpu(), t.tensor())
        assert (counts if apart else refs).tolist() == want
        assert not apart or refs.tolist() == t.refs


# one column into the second turn, its middle, a third turn, and a table that ends with the second
@pytest.mark.parametrize("pages,mb", [(4097, 4097), (4375, 4600), (8500, 9000), (8192, 8192), (4104, 5000)])
def test_fork(pages, mb):
    longest = pages * 16 - 3
    t = Table([longest, longest - 1000, 100, 66000 if pages > 4200 else 30000, 0], {1: (0, pages - 70), 3: (1, 1500)}, mb, 10, pages)
    # taken over whole, cut inside each turn, shared by several, dropped
    check_fork(t, [0, 0, 1, 3, -1, 2, 2], None)
    check_fork(t, [0, 0, 1, 1, 3], [longest - 40, 65600, 65536, 65537, 20])
    check_fork(t, [1], [longest - 2000])
    check_fork(t, [-1, 2], None)


@pytest.mark.parametrize("S,N", [(2100, 2100), (4090, 7), (5, 4200)])
def test_fork_of_more_rows_than_are_fetched_together(S, N):
    """Origins are fetched again in every turn where both tables have more than 4096 rows together."""
    r = random.Random(S)
    lens = [69000, 67000, 5] + [r.choice([0, 16, r.randint(1, 400)]) for _ in range(S - 4)] + [66001]
    t = Table(lens, {1: (0, 4150), S - 1: (0, 4100), **{i: (i - 1, r.randint(0, 20)) for i in range(4, S - 1, 3) if lens[i - 1] > 320}}, 4500, 10, S)
    src = [r.choice([-1, r.randrange(S), r.randrange(S)]) for _ in range(N)]
    src[0], src[N // 2], src[-1] = 0, S - 1, 1
    check_fork(t, src, None)
    keep = [r.choice([10 ** 9, r.randint(0, 500)]) for _ in range(N)]
    keep[0], keep[N // 2] = 68000, 10 ** 9
    check_fork(t, src, keep)


@pytest.mark.parametrize("apart", [False, True])
def test_append_and_compact(apart):
    """A row of several workgroups' worth of table entries grows past a turn's columns; then the holes between all pages are filled."""
    t = Table([70005, 66007, 66007, 9], {1: (0, 4000), 2: (1, 4126)}, 4600, 500, 3)
    cu = [0, 3000, 3001, 3002, 3002]
    caches = new_caches(t.nb, 1, 8, torch.bfloat16, 2)
    before, status = caches.clone(), ints([0])
    ins = [t.tensor().to(DEV), ints(t.lens), ints(t.refs)]
    outs = [torch.full_like(x, JUNK) for x in ins] if apart else ins
    binding.hook_pages_append(ints(cu), *ins, caches, status, block_table_out=outs[0], seq_lens_out=outs[1], ref_counts_out=outs[2])
    rows, L, counts, copies, bits = G.append(cu, t.short(), t.lens, t.refs)
    assert bits == 0 and int(status) == 0 and copies and outs[1].tolist() == L and outs[2].tolist() == counts
    assert torch.equal(outs[0].cpu(), as_tensor(rows, t.mb))
    for a, b, n in copies:
        before[:, b, :, :n] = before[:, a, :, :n]
    assert torch.equal(caches, before)

    page_map, live = ints([55] * t.nb), ints([0])
    table, refs = outs[0], outs[2]
    to = [torch.full_like(table, JUNK), torch.full_like(refs, 5)] if apart else [table, refs]
    binding.hook_pages_compact(table, outs[1], refs, caches, page_map, live, status, block_table_out=to[0], ref_counts_out=to[1])
    wide = [rows[0] + [JUNK] * (t.mb - len(rows[0]))] + rows[1:]
    rows, counts, want_map, n, moves, bits = G.compact(wide, L, counts)
    assert bits == 0 and int(status) == 0 and moves and int(live) == n and page_map.tolist() == want_map and to[1].tolist() == counts
    assert torch.equal(to[0].cpu(), as_tensor(rows, t.mb))
    for a, b in moves:
        before[:, b] = before[:, a]
    assert torch.equal(caches, before)
