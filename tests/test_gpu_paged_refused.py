"""Where free pages run out: sequences that got no room store nothing, keep their lengths and see their own rows only, with nothing read back
by the host in between."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from paged import DEV, PAGES, ints, slots_of, table_of
from test_gpu_paged_append import normed, weights
from test_gpu_pages import Pool
from test_gpu_prompt_attn import ROWS, offsets, randn, starts
from test_gpu_rotary import cache, close, inputs, turned

pytestmark = pytest.mark.gpu


def attention(Qr, pool, new, table, lens, most):
    total, Hq, D = Qr.shape
    O = torch.empty_like(Qr)
    n = l2kv.l2kv_paged_attn_workspace_bytes(len(new), Hq, pool.Kc.shape[0], total, most, D, Qr.dtype)
    l2kv.l2kv_paged_attn(Qr, pool.Kc, pool.Vc, offsets(new), table, pool.page, lens, most, O, torch.empty(max(1, n), dtype=torch.uint8, device=DEV))
    return O


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("spare,given", [(0, [20, 20, 20]), (1, [21, 20, 20]), (2, [21, 21, 21])])
def test_branches_of_one_page(dtype, D, spare, given):
    """Three branches of 20 rows with both pages in common want one token more: who gets no copy leaves the page as it is."""
    Hq, Hkv, page = 4, 2, 16
    p = Pool(2 + spare, page, Hkv, D, dtype)
    t = p.init(1, 3)
    p.reserve(t, [0], [20])
    b, lens = p.fork(t, [20], [0, 0, 0])
    p.release(t, [0])
    ends = torch.empty(3, dtype=torch.int32, device=DEV)
    l2kv.l2kv_pages_reserve(b, ints(lens), ints([21] * 3), ends, p.refs, p.free, p.count, page, p.Kc, p.Vc, p.norms, p.pos, p.ws)
    assert ends.tolist() == given
    slots = [slots_of(row, 21, page).to(DEV) for row in b.tolist()]
    held = [[x[:, at[:20]].clone() for x in (p.Kc, p.Vc, p.norms, p.pos)] for at in slots]
    Q, K, V = inputs(1, 3, Hq, Hkv, D, dtype)
    (qw, kw), positions, freqs = weights(2, D), ints([20, 20, 20]), l2kv.l2kv_rotary_freqs(D).to(DEV)
    Qr, lens_out = torch.empty((3, Hq, D), dtype=dtype, device=DEV), ints([0] * 3)
    # the first layer's call says where sequences end, those of further layers need not
    for out in (lens_out, None):
        l2kv.l2kv_paged_append_reserved(Q, K, V, positions, freqs, Qr, p.Kc, p.Vc, p.norms, p.pos, offsets([1] * 3), b, page, ints(lens), ends, out, qw, kw)
    assert lens_out.tolist() == given
    O = attention(Qr, p, [1] * 3, b, lens_out, 21)
    want = turned(normed(K, kw, 1e-6), positions, freqs, 0, 1.0)
    close(Qr, turned(normed(Q, qw, 1e-6), positions, freqs, 0, 1.0))
    for s, (at, n) in enumerate(zip(slots, given)):
        for x, y in zip((p.Kc, p.Vc, p.norms, p.pos), held[s]):
            assert torch.equal(x[:, at[:20]], y)
        if n == 21:
            close(p.Kc[:, at[20]][None], want[s][None])
            assert torch.equal(p.Vc[:, at[20]], V[s])
        rows = at[:n]
        check(O[s:s + 1], attend(Qr[s:s + 1], p.Kc[:, rows], p.Vc[:, rows], torch.ones((1, n), dtype=torch.bool, device=DEV)), n)


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_ends_anywhere(page, dtype, D):
    """Before the first new row and behind the last, inside of pages and between them, beyond the table, and with pages that are missing."""
    new, have = [40, 3, 600, 1, 1, 300, 70, 5], [10, 15, 3, 700, 0, 255, 0, 9]
    ends = [31, 100000, 517, 700, 1, 100, -5, 9]
    total, Hq, Hkv = sum(new), 3, 2
    table, n_pages, slots = table_of([h + n for h, n in zip(have, new)], page, 3)
    table[2][300 // page] = -1                                     # before its end
    table[5][300 // page] = n_pages                                # behind it
    Q, K, V = inputs(5, total, Hq, Hkv, D, dtype)
    (qw, kw), positions, freqs = weights(2, D), torch.arange(total, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(32).to(DEV)
    Qr = torch.empty((total, Hq, D), dtype=dtype, device=DEV)
    Kc, Vc, norms, pos = cache(Hkv, n_pages * page, D, dtype)
    lens_out = ints([-1] * len(new))
    l2kv.l2kv_paged_append_reserved(Q, K, V, positions, freqs, Qr, Kc, Vc, norms, pos, offsets(new), ints(table), page, ints(have), ints(ends), lens_out, qw, kw)
    close(Qr, turned(normed(Q, qw, 1e-6), positions, freqs, 0, 1.0))
    to, tokens, lens = [], [], []
    for s, first in enumerate(starts(new)[:-1]):
        there = [r < ends[s] and 0 <= table[s][r // page] < n_pages for r in range(have[s], have[s] + new[s])]
        lens.append(have[s] + (there + [False]).index(False))
        tokens += [first + j for j, x in enumerate(there) if x]
        to += [int(slots[s][have[s] + j]) for j, x in enumerate(there) if x]
    assert lens_out.tolist() == lens
    to, tokens = torch.tensor(to, device=DEV), torch.tensor(tokens, device=DEV)
    close(Kc[:, to].transpose(0, 1), turned(normed(K, kw, 1e-6), positions, freqs, 0, 1.0)[tokens])
    assert torch.equal(Vc[:, to], V[tokens].transpose(0, 1)) and torch.equal(pos[:, to], positions[tokens].expand(Hkv, -1))
    rest = torch.ones(n_pages * page, dtype=torch.bool, device=DEV)
    rest[to] = False
    for x in (Kc, Vc, norms, pos):
        assert (x[:, rest] == 9).all()


def test_without_ends_and_with_ends_at_the_lengths():
    """No ends make it l2kv_paged_append; lengths for ends store nothing."""
    new, have, page, D = [5, 40], [3, 20], 16, 64
    table, n_pages, _ = table_of([8, 60], page, 1)
    Q, K, V = inputs(7, 45, 2, 1, D, torch.float32)
    positions, freqs, lens_in, results = torch.arange(45, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(D).to(DEV), ints(have), []
    for call, more in ((l2kv.l2kv_paged_append, ()), (l2kv.l2kv_paged_append_reserved, (None,)), (l2kv.l2kv_paged_append_reserved, (lens_in,))):
        Qr, c, lens_out = torch.empty((45, 2, D), device=DEV), cache(1, n_pages * page, D, torch.float32), ints([0, 0])
        call(Q, K, V, positions, freqs, Qr, *c, offsets(new), ints(table), page, lens_in, *more, lens_out)
        results.append((Qr, lens_out, *c))
    for a, b in zip(results[0], results[1]):
        assert torch.equal(a, b)
    assert torch.equal(results[0][0], results[2][0]) and results[2][1].tolist() == have and all((x == 9).all() for x in results[2][2:])


def test_a_captured_loop_that_runs_out():
    """A decode step captured once and replayed until the pages are gone: sequences stop one after the other, at their last page's end, and
    what they hold stays as it was."""
    page, Hq, Hkv, D, n = 16, 4, 2, 64, 3
    p = Pool(7, page, Hkv, D, torch.bfloat16)
    t, start = p.init(n, 5), [30, 16, 1]
    p.reserve(t, [0] * n, start)                                   # 2 + 1 + 1 pages; three are left
    qkv = randn(torch.Generator(device=DEV).manual_seed(1), n, Hq + 2 * Hkv, D).bfloat16()
    lens, to, ends, out, freqs, off = ints(start), ints([0] * n), ints([0] * n), ints([0] * n), l2kv.l2kv_rotary_freqs(D).to(DEV), offsets([1] * n)
    Qr, O = (torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = torch.empty(max(1, l2kv.l2kv_paged_attn_workspace_bytes(n, Hq, Hkv, n, 80, D, torch.bfloat16)), dtype=torch.uint8, device=DEV)

    def step():
        torch.add(lens, 1, out=to)
        l2kv.l2kv_pages_reserve(t, lens, to, ends, p.refs, p.free, p.count, page, p.Kc, p.Vc, p.norms, p.pos, p.ws)
        l2kv.l2kv_paged_append_reserved(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], lens, freqs, Qr, p.Kc, p.Vc, p.norms, p.pos, off, t, page, lens,
                                        ends, out)
        l2kv.l2kv_paged_attn(Qr, p.Kc, p.Vc, off, t, page, out, 80, O, ws)
        lens.copy_(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    host, want = t.tolist(), list(start)
    for i in range(45):
        qkv.copy_(randn(torch.Generator(device=DEV).manual_seed(10 + i), *qkv.shape))
        held = [p.Vc[:, slots_of(row, m, page).to(DEV)].clone() for row, m in zip(host, want)]
        p.model.reserve(host, want, [m + 1 for m in want])
        graph.replay()
        torch.cuda.synchronize()
        more = [m + 1 if m % page or host[s][m // page] >= 0 else m for s, m in enumerate(want)]
        assert lens.tolist() == more and t.tolist() == host
        for s, (old, m) in enumerate(zip(want, more)):
            at = slots_of(host[s], m, page).to(DEV)
            assert torch.equal(p.Vc[:, at[:old]], held[s])
            if m > old:
                assert torch.equal(p.Vc[:, at[old]], qkv[s, Hq + Hkv:])
            check(O[s:s + 1], attend(Qr[s:s + 1], p.Kc[:, at], p.Vc[:, at], torch.ones((1, m), dtype=torch.bool, device=DEV)), m)
        want = more
    assert int(p.count) == 0 and want == [48, 32, 32]


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("spare,served", [(4, [True, False, False]), (2, [False, False, False]), (7, [True, True, True]), (6, [True, True, False])])
def test_a_compaction_that_gets_no_room(dtype, D, spare, served):
    """The ends of the reservation are what is kept: sequences that got no room keep nothing in the new table and all in the old one, and go on
    from it, a token each."""
    page, Hq, Hkv, have, want = 16, 4, 2, [90, 64, 40], [45, 32, 20]
    p = Pool(6 + 4 + 3 + spare, page, Hkv, D, dtype)
    t = p.init(3, 7)
    p.reserve(t, [0] * 3, have)
    cache = (p.Kc, p.Vc, p.norms, p.pos)
    p.norms.square_()
    lens, keep, zero, ends, lens_new, out = ints(have), ints(want), ints([0] * 3), ints([0] * 3), ints([0] * 3), ints([0] * 3)
    new = torch.full_like(t, -1)
    old = [slots_of(row, n, page).to(DEV) for row, n in zip(t.tolist(), have)]
    was = [x.clone() for x in cache]

    def reserve(table, first, to):
        l2kv.l2kv_pages_reserve(table, first, to, ends, p.refs, p.free, p.count, page, *cache, p.ws)
    reserve(new, zero, keep)
    ws = torch.empty(l2kv.l2kv_paged_compress_workspace_bytes(Hkv, 3, sum(have), sum(want)), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_paged_compress(*cache, t, lens, ends, new, lens_new, page, sum(have), sum(want), max(have), ws)
    there = ends == keep
    l2kv.l2kv_pages_release(t, torch.where(there, 0, lens).int(), p.refs, p.free, p.count, page, p.ws)
    table, lens = torch.where(there[:, None], new, t), torch.where(there, lens_new, lens).int()
    # one more token of each; what compaction gave back is enough for it where there was a compaction
    reserve(table, lens, lens + 1)
    Q, K, V = inputs(3, 3, Hq, Hkv, D, dtype)
    Qr, freqs = torch.empty((3, Hq, D), dtype=dtype, device=DEV), l2kv.l2kv_rotary_freqs(D).to(DEV)
    l2kv.l2kv_paged_append_reserved(Q, K, V, lens, freqs, Qr, *cache, offsets([1] * 3), table, page, lens, ends, out)
    O = attention(Qr, p, [1] * 3, table, out, 91)

    assert there.tolist() == served and lens_new.tolist() == [w if x else 0 for w, x in zip(want, served)]
    before = [w if x else h for h, w, x in zip(have, want, served)]
    assert lens.tolist() == before and out.tolist() == [n + 1 for n in before]
    for s, n in enumerate(before):
        at = slots_of(table[s].tolist(), n + 1, page).to(DEV)
        for h in range(Hkv):
            rows = old[s]
            if served[s]:
                rows = rows[torch.sort(was[2][h, rows], stable=True).indices[:n].sort().values]
            for x, y in zip(cache, was):
                assert torch.equal(x[h, at[:n]], y[h, rows])
        assert torch.equal(p.Vc[:, at[n]], V[s])
        check(O[s:s + 1], attend(Qr[s:s + 1], p.Kc[:, at], p.Vc[:, at], torch.ones((1, n + 1), dtype=torch.bool, device=DEV)), n + 1)
