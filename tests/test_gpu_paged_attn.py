"""Attention over a cache in pages against its definition in 64 bits, rows gathered through the table on the host."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from paged import DEV, PAGES, ints, slots_of, table_of
from test_gpu_prompt_attn import LENGTHS, ROWS, offsets, randn, starts

pytestmark = pytest.mark.gpu


class Case:
    """Sequences with `rows` rows, of which the last `new` are queried; whatever is no row of a sequence holds NaN."""

    def __init__(self, seed, new, rows, Hq, Hkv, D, dtype, page):
        self.new, self.rows, self.page = new, rows, page
        self.table, self.n_pages, self.slots = table_of(rows, page, seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        held = torch.cat(self.slots).to(DEV)
        self.Kc, self.Vc = (torch.full((Hkv, self.n_pages * page, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
        self.Kc[:, held] = (randn(gen, Hkv, len(held), D) * torch.exp(0.5 * randn(gen, Hkv, len(held), 1))).to(dtype)
        self.Vc[:, held] = randn(gen, Hkv, len(held), D).to(dtype)
        self.Q = randn(gen, sum(new), Hq, D).to(dtype)

    def workspace(self, top):
        n = l2kv.l2kv_paged_attn_workspace_bytes(len(self.new), self.Q.shape[1], self.Kc.shape[0], len(self.Q), top, self.Q.shape[2], self.Q.dtype)
        return torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)

    def run(self, scale=0.0, top=None, Q=None, **kw):
        top = top or max(1, max(self.rows))
        O = torch.full(self.Q.shape, float("nan"), dtype=self.Q.dtype, device=DEV)
        l2kv.l2kv_paged_attn(self.Q if Q is None else Q, self.Kc, self.Vc, offsets(self.new), ints(self.table), self.page, ints(self.rows), top, O,
                             self.workspace(top), scale, **kw)
        return O

    def verify(self, O, scale=None, some=None):
        q = starts(self.new)
        for s, (n, m) in enumerate(zip(self.new, self.rows)):
            if some is not None and s not in some:
                continue
            at = self.slots[s].to(DEV)
            seen = torch.arange(m, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + m - n
            where = slice(q[s], q[s + 1])
            check(O[where], attend(self.Q[where], self.Kc[:, at], self.Vc[:, at], seen, scale), m)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("G", [1, 3, 4])
@pytest.mark.parametrize("new,rows", LENGTHS)
@pytest.mark.parametrize("page", [16, 64])
def test_lengths(dtype, D, G, new, rows, page):
    c = Case(len(new) + D, new, rows, 2 * G, 2, D, dtype, page)
    c.verify(c.run())


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([1, 1, 1, 1, 1], [1, 15, 16, 17, 700]), ([1] * 70, [(37 * i) % 300 for i in range(70)]),
                                      ([1, 0, 1, 1], [5000, 9, 0, 4097]), ([1], [20011]), ([4, 1, 9], [3000, 64, 9])])
def test_single_tokens_and_few(page, dtype, D, new, rows):
    """Decode steps: one token a sequence, as a rule, from no row to many, few sequences and many."""
    c = Case(page + len(new), new, rows, 8, 2, D, dtype, page)
    first = c.run()
    c.verify(first)
    assert torch.equal(first, c.run())


@pytest.mark.parametrize("G", [1, 2, 5, 6, 7, 8])
@pytest.mark.parametrize("new,rows", [([1, 7], [90, 7]), ([200, 61], [200, 700]), ([1] * 40, [333] * 40)])
@pytest.mark.parametrize("page", [16, 256])
def test_groups(G, new, rows, page):
    c = Case(G, new, rows, 3 * G, 3, 128, torch.bfloat16, page)
    c.verify(c.run())


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([150], [9001]), ([700], [700]), ([1500, 0, 777, 2, 1], [1500, 0, 1777, 2, 3001])])
@pytest.mark.parametrize("page", [16, 128])
def test_chunks(dtype, D, new, rows, page):
    c = Case(7, new, rows, 8, 2, D, dtype, page)
    c.verify(c.run())


@pytest.mark.parametrize("n_seq", [64, 65, 1000, 1025, 4097])
@pytest.mark.parametrize("most", [1, 3])
def test_many_sequences(n_seq, most):
    gen = torch.Generator().manual_seed(n_seq)
    new = torch.randint(0, most + 1, (n_seq,), generator=gen).tolist() if most > 1 else [1] * n_seq
    rows = [n + h for n, h in zip(new, torch.randint(0, 90, (n_seq,), generator=gen).tolist())]
    rows[n_seq // 2] = 700
    c = Case(n_seq, new, rows, 4, 2, 64, torch.bfloat16, 16)
    O = c.run()
    assert torch.isfinite(O.float()).all()
    c.verify(O, some=set([0, 1, n_seq // 2, n_seq - 2, n_seq - 1] + list(range(2, n_seq, 97))))


@pytest.mark.parametrize("dtype,D", ROWS)
def test_like_prompt_attention(dtype, D):
    """Pages in the order of a plane are that plane: the same bits as l2kv_prompt_attn where every item has a workgroup for itself (shares of items
    are cut elsewhere), queries from a projection."""
    n, page, Hkv, Hq = 300, 32, 2, 4
    new, rows = [12 - s % 3 for s in range(n)], [64] * n
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V = (randn(gen, Hkv, sum(rows), D).to(dtype) for _ in range(2))
    Q = randn(gen, sum(new), 3 * Hq, D).to(dtype)[:, Hq:2 * Hq]
    a, b = (torch.empty((sum(new), Hq, D), dtype=dtype, device=DEV) for _ in range(2))
    sizes = (n, Hq, Hkv, sum(new), 64, D, dtype)
    assert l2kv.l2kv_prompt_attn_workspace_bytes(*sizes) == l2kv.l2kv_paged_attn_workspace_bytes(*sizes) == 0
    l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), offsets(rows), None, 64, a, None, 0.3)
    table = [[2 * s, 2 * s + 1] for s in range(n)]
    l2kv.l2kv_paged_attn(Q, K, V, offsets(new), ints(table), page, ints(rows), 64, b, None, 0.3)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_that_are_not_finite(dtype, D, new, bad):
    """They reach the queries that see them and no other."""
    c = Case(3, [new, new], [190, 300], 4, 2, D, dtype, 16)
    clean = c.run()
    c.Vc[:, c.slots[0][70], 5] = bad                      # seen by all queries of the first sequence
    got = c.run()
    assert torch.equal(got[new:], clean[new:])
    assert (got[:new, :, 5].isnan() if bad != bad else got[:new, :, 5] == bad).all()
    others = [d for d in range(D) if d != 5]
    assert torch.equal(got[:new][..., others], clean[:new][..., others])


def test_shared_pages_and_entries_that_are_none():
    """Two sequences with the same beginning; numbers outside the pages are forced into them; tokens behind the last sequence stay."""
    c = Case(4, [2, 1], [100, 80], 4, 2, 128, torch.bfloat16, 16)
    c.table[1][:3] = c.table[0][:3]
    c.slots[1] = slots_of(c.table[1], 80, 16)
    c.verify(c.run())
    table = [row[:] for row in c.table]
    for entry, page in ((-5, 0), (1 << 30, c.n_pages - 1)):
        table[0][1] = entry
        c.table[0][1] = page
        c.slots[0] = slots_of(c.table[0], 100, 16)
        c.Kc.nan_to_num_(1.0), c.Vc.nan_to_num_(1.0)
        O = torch.full((5, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        Q = torch.cat([c.Q, c.Q[:2]])
        l2kv.l2kv_paged_attn(Q, c.Kc, c.Vc, offsets(c.new), ints(table), 16, ints(c.rows), 100, O, c.workspace(100))
        c.verify(O[:3])
        assert (O[3:] == 7).all()


def test_lengths_beyond_the_table_and_the_bound():
    """More rows than a sequence has pages for count as that many; max_kv sizes the cut only."""
    c = Case(8, [3, 1], [5000, 900], 4, 2, 128, torch.bfloat16, 16)
    for top in (1, 600, 2000):
        c.verify(c.run(top=top))
    c = Case(9, [3, 2], [64, 48], 4, 2, 64, torch.float32, 16)
    c.table = [row[:4] for row in c.table]
    c.table[1][3] = c.table[0][0]
    O = torch.empty_like(c.Q)
    l2kv.l2kv_paged_attn(c.Q, c.Kc, c.Vc, offsets(c.new), ints(c.table), 16, ints([1 << 30, 1000]), 64, O, c.workspace(64))
    c.rows, c.slots = [64, 64], [slots_of(t, 64, 16) for t in c.table]
    c.verify(O)
    l2kv.l2kv_paged_attn(c.Q, c.Kc, c.Vc, offsets(c.new), ints(c.table), 16, ints([-3, 0]), 64, O, c.workspace(64))
    assert (O == 0).all()


def test_far_pages():
    """Slots whose place passes 32 bits, in elements and in bytes."""
    page, D, n_pages = 256, 128, (1 << 16) + 40
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V = (torch.empty((1, n_pages * page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rows = 700
    entries = [n_pages - 1, 3, n_pages - 2]
    at = slots_of(entries, rows, page).to(DEV)
    K[:, at], V[:, at] = randn(gen, 1, rows, D).bfloat16(), randn(gen, 1, rows, D).bfloat16()
    for n in (1, 20):
        Q = randn(gen, n, 2, D).bfloat16()
        O = torch.empty_like(Q)
        ws = torch.empty(max(1, l2kv.l2kv_paged_attn_workspace_bytes(1, 2, 1, n, rows, D, torch.bfloat16)), dtype=torch.uint8, device=DEV)
        l2kv.l2kv_paged_attn(Q, K, V, offsets([n]), ints([entries]), page, ints([rows]), rows, O, ws)
        seen = torch.arange(rows, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + rows - n
        check(O, attend(Q, K[:, at], V[:, at], seen), rows)


def test_streams_and_graphs():
    """A call on another stream, and graphs that share a workspace, replayed in turn on fresh inputs, tables and lengths."""
    shapes = [([1, 1], [3000, 60]), ([2, 5], [3000, 60]), ([300], [300])]
    ws = torch.zeros(max(l2kv.l2kv_paged_attn_workspace_bytes(len(n), 4, 2, sum(n), max(r), 128, torch.bfloat16) for n, r in shapes),
                     dtype=torch.uint8, device=DEV)
    side, held = torch.cuda.Stream(), []
    for new, rows in shapes:
        c = Case(1, new, rows, 4, 2, 128, torch.bfloat16, 32)
        O, q, t, lens = torch.empty_like(c.Q), offsets(new), ints(c.table), ints(rows)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            l2kv.l2kv_paged_attn(c.Q, c.Kc, c.Vc, q, t, 32, lens, max(rows), O, ws)
        torch.cuda.current_stream().wait_stream(side)
        c.verify(O)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            l2kv.l2kv_paged_attn(c.Q, c.Kc, c.Vc, q, t, 32, lens, max(rows), O, ws)
        held.append((graph, c, O, t, lens, new, rows, q))
    for round_ in range(3):
        for graph, c, O, t, lens, new, rows, q in held:
            fresh = Case(50 + round_, new, [max(r - 7 * round_, n) for r, n in zip(rows, new)], 4, 2, 128, torch.bfloat16, 32)
            fresh.table = [row + [-1] * (t.shape[1] - len(row)) for row in fresh.table]
            slots = fresh.Kc.shape[1]
            c.Q.copy_(fresh.Q), c.Kc[:, :slots].copy_(fresh.Kc), c.Vc[:, :slots].copy_(fresh.Vc)
            t.copy_(ints(fresh.table)), lens.copy_(ints(fresh.rows))
            O.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            fresh.verify(O)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([300, 120], [7000, 1500]), ([700], [9000]), ([40, 1, 350, 0, 90], [6000, 5000, 350, 9, 4444])])
@pytest.mark.parametrize("G,Hkv", [(4, 4), (2, 1)])
def test_chunks_in_stretches(dtype, D, new, rows, G, Hkv):
    """Few chunks over many rows: equal stretches of wide blocks, which begin and end inside of items."""
    c = Case(17, new, rows, G * Hkv, Hkv, D, dtype, 32)
    first = c.run()
    c.verify(first)
    assert torch.equal(first, c.run())


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([3, 0, 0], [1, 5, 5]), ([2, 0, 1, 0], [300, 40, 7, 0]), ([0, 3, 0, 1, 0], [9, 4000, 0, 2500, 1]), ([0, 0, 1], [5, 0, 1])])
def test_few_tokens_of_many_sequences(dtype, D, new, rows):
    """No more tokens than sequences: some have several, some none, some more than rows; queries from a projection."""
    c = Case(23, new, rows, 4, 2, D, dtype, 16)
    both = torch.cat([c.Q, c.Q.flip(0), c.Q * 3], 1)
    c.verify(c.run(Q=both[:, :4]))


def test_scale_and_no_workspace():
    c = Case(2, [1, 1], [45, 300], 2, 2, 64, torch.float32, 16)
    O = torch.empty_like(c.Q)
    l2kv.l2kv_paged_attn(c.Q, c.Kc, c.Vc, offsets(c.new), ints(c.table), 16, ints(c.rows), 300, O, None, 0.7)
    c.verify(O, scale=0.7)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("rows", [[700, 40, 9, 300, 1, 60], [5000, 40, 9, 3000, 1, 60]])
def test_padded_single_tokens_any_distance_apart(dtype, D, rows):
    """A batch of single tokens with sequences that have none, fewer tokens than the buffers, queries out of wider rows, lengths beyond the bound."""
    new = [1, 0, 0, 1, 0, 1]
    c = Case(31, new, rows, 4, 2, D, dtype, 16)
    wide = torch.full((5, 7, D), float("nan"), dtype=dtype, device=DEV)
    wide[:3, 2:6] = c.Q
    for top in (max(rows), 600):
        O = torch.full((5, 4, D), 7.0, dtype=dtype, device=DEV)
        ws = torch.full((l2kv.l2kv_paged_attn_workspace_bytes(6, 4, 2, 5, top, D, dtype),), 0xff, dtype=torch.uint8, device=DEV)
        l2kv.l2kv_paged_attn(wide[:, 2:6], c.Kc, c.Vc, offsets(new), ints(c.table), 16, ints(rows), top, O, ws)
        c.verify(O[:3])
        assert (O[3:] == 7).all()
