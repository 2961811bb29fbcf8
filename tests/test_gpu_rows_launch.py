"""Attention of many query rows under every way its work is cut: blocks of 256, 128 and 64 rows, a workgroup for each item or equal
stretches of all of them, few sequences and very many.  The reference is the definition in 64 bits."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from test_gpu_prompt_attn import DEV, ROWS, make, offsets, randn, run, starts, verify, workspace
from test_gpu_tree_attn import Case, ints

pytestmark = pytest.mark.gpu


def lengths(n, top, seed, empty=0.3):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randint(1, top + 1, (n,), generator=gen)
    return (x * (torch.rand(n, generator=gen) >= empty)).tolist()


# sequences on both sides of a wave's 64 and of 64 * 64, most of them short and some empty, also at both ends
@pytest.mark.parametrize("n_seq", [63, 64, 65, 128, 1000, 1024, 1025, 4096, 4097, 5000])
@pytest.mark.parametrize("fresh", [True, False])
def test_many_sequences_of_a_prompt(n_seq, fresh):
    new = lengths(n_seq, 5, n_seq)
    new[0], new[-1], new[n_seq // 2] = 0, 0, 70
    rows = list(new) if fresh else [n + h for n, h in zip(new, lengths(n_seq, 9, n_seq + 1))]
    Q, K, V = make(n_seq, new, rows, 4, 2, 64, torch.bfloat16)
    O = run(Q, K, V, new, rows).cpu()
    Q, K, V = Q.cpu(), K.cpu(), V.cpu()
    q, k = starts(new), starts(rows)
    some = [0, 1, 2, n_seq // 2 - 1, n_seq // 2, n_seq // 2 + 1, n_seq - 2, n_seq - 1] + list(range(3, n_seq, 97))
    assert torch.isfinite(O.float()).all()                              # every token has been written
    for s in some:
        i = torch.arange(new[s])[:, None]
        seen = torch.arange(rows[s])[None] <= i + rows[s] - new[s]
        where = slice(q[s], q[s + 1])
        check(O[where], attend(Q[where], K[:, k[s]:k[s + 1]], V[:, k[s]:k[s + 1]], seen, None), rows[s])


@pytest.mark.parametrize("n_seq", [65, 1024, 1025, 4097])
def test_many_trees(n_seq):
    nodes, lens = lengths(n_seq, 4, n_seq), lengths(n_seq, 40, n_seq + 1)
    nodes[-1], nodes[0], lens[3] = 2, 0, 700
    c = Case(n_seq, nodes, lens, 4, 2, 64, torch.bfloat16, words=1)
    O = c.run()
    assert torch.isfinite(O.float()).all()
    q, k = starts(nodes), starts(c.room)
    for s in [0, 1, 2, 3, n_seq - 2, n_seq - 1] + list(range(4, n_seq, 131)):
        a, b = slice(q[s], q[s + 1]), slice(k[s], k[s] + lens[s])
        seen = torch.cat([torch.ones((nodes[s], lens[s]), dtype=torch.bool), c.masks[s].bool()], 1).to(DEV)
        want = attend(c.Q[a], torch.cat([c.Kc[:, b], c.Kt[:, a]], 1), torch.cat([c.Vc[:, b], c.Vt[:, a]], 1), seen, None)
        check(O[a], want, lens[s] + nodes[s])


# few long items: stretches that cut an item into many parts, that hold the end of one and the beginning of the next, with items of length
# zero between them; blocks of every width, of which the last is not full
@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([17], [6000]), ([40], [5000]), ([100], [9001]), ([10, 1, 0, 3], [3000, 1, 0, 4097]), ([30, 33], [0, 8000]),
                                      ([3, 90, 2], [2500, 3333, 2501]), ([9, 70], [4, 7000])])
@pytest.mark.parametrize("G", [1, 4])
def test_stretches(dtype, D, new, rows, G):
    Hkv = 2
    Q, K, V = make(len(new) + D, new, rows, Hkv * G, Hkv, D, dtype)
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("n_seq,n,have", [(300, 12, 0), (300, 40, 30), (130, 64, 0), (520, 3, 200)])
def test_an_item_for_each_workgroup(dtype, D, n_seq, n, have):
    new = [n - s % 3 for s in range(n_seq)]
    rows = [x + have for x in new]
    Q, K, V = make(n_seq + n, new, rows, 8, 2, D, dtype)
    O = run(Q, K, V, new, rows)
    q, k = starts(new), starts(rows)
    assert torch.isfinite(O.float()).all()
    for s in range(0, n_seq, 23):
        i = torch.arange(new[s], device=DEV)[:, None]
        seen = torch.arange(rows[s], device=DEV)[None] <= i + have
        where = slice(q[s], q[s + 1])
        check(O[where], attend(Q[where], K[:, k[s]:k[s + 1]], V[:, k[s]:k[s + 1]], seen, None), rows[s])


@pytest.mark.parametrize("dtype,D", ROWS)
def test_the_widest_block(dtype, D):
    """A prompt long enough for blocks of 256 rows with a workgroup each; its ends and some places between are looked at."""
    n = 17600
    Q, K, V = make(1, [n], [n], 8, 4 if D < 256 else 2, D, dtype)
    O = run(Q, K, V, [n], [n])
    for first in (0, 31, 100, 2040, n // 2 - 3, n - 70):
        i = torch.arange(first, first + 70, device=DEV)
        top = first + 70
        seen = torch.arange(top, device=DEV)[None] <= i[:, None]
        check(O[first:top], attend(Q[first:top], K[:, :top], V[:, :top], seen, None), top)


def test_a_bound_above_the_lengths_has_no_effect_on_the_result():
    """The bound chooses how the work is cut, the arrays say what it is."""
    new, rows = [20, 3, 0, 60], [700, 3, 5, 60]
    Q, K, V = make(5, new, rows, 8, 2, 128, torch.bfloat16)
    for top in (1, 60, 700, 768):
        O = torch.full_like(Q, float("nan"))
        l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), offsets(rows), None, top, O, workspace(4, 8, 2, Q.shape[0], top, 128, Q.dtype))
        verify(O, Q, K, V, new, rows)


def test_tokens_behind_the_last_sequence_are_left():
    for new, rows in (([5, 9], [4000, 300]), ([300, 200], [300, 200]), ([2], [9])):
        Q, K, V = make(9, new + [7], rows + [7], 8, 2, 128, torch.bfloat16)
        O = torch.full_like(Q, 3.0)
        l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), offsets(rows), None, max(rows), O, workspace(len(new), 8, 2, Q.shape[0], max(rows), 128, Q.dtype))
        n = sum(new)
        assert (O[n:] == 3).all()
        verify(O[:n], Q[:n], K, V, new, rows)


def test_two_streams_and_replays_with_a_workspace_each():
    """Two calls that run at the same time, captured and replayed between eager ones: the same bits as alone."""
    cases = []
    for seed, new, rows in ((1, [6], [9000]), (2, [50, 20], [5000, 3000])):
        Q, K, V = make(seed, new, rows, 8, 2, 128, torch.bfloat16)
        cases.append((Q, K, V, offsets(new), offsets(rows), max(rows), workspace(len(new), 8, 2, Q.shape[0], max(rows), 128, Q.dtype), torch.empty_like(Q)))

    def call(c, stream=None):
        l2kv.l2kv_prompt_attn(*c[:5], None, c[5], c[7], c[6], stream=stream)
    want = []
    for c in cases:
        call(c)
        want.append(c[7].clone())
    torch.cuda.synchronize()
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(c)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for c in cases:
            c[7].zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c[7], w) for c, w in zip(cases, want))
        for c, s in zip(cases, streams):
            call(c, s)
        torch.cuda.synchronize()
        assert all(torch.equal(c[7], w) for c, w in zip(cases, want))


def test_far_planes():
    """Heads more than 2^32 bytes apart, and rows at the far end of one, cut into stretches."""
    rows, D = 1 << 23, 128
    K = torch.empty((3, rows, D), dtype=torch.bfloat16, device=DEV)
    V = torch.empty((3, rows, D), dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(0)
    n, at = 3000, rows - 3001
    K[:, at:at + n], V[:, at:at + n] = randn(gen, 3, n, D).to(K.dtype), randn(gen, 3, n, D).to(K.dtype)
    Q = randn(gen, 4, 6, D).to(K.dtype)
    O = torch.empty_like(Q)
    off = torch.tensor([at, at + n], device=DEV)
    l2kv.l2kv_prompt_attn(Q, K, V, offsets([4]), off, None, n, O, workspace(1, 6, 3, 4, n, D, Q.dtype))
    verify(O, Q, K[:, at:at + n], V[:, at:at + n], [4], [n])
    mask = ints([1, 3, 5, 15]).view(4, 1)
    Kt, Vt = randn(gen, 3, 4, D).to(K.dtype), randn(gen, 3, 4, D).to(K.dtype)
    ws = torch.full((l2kv.l2kv_tree_attn_workspace_bytes(1, 6, 3, 4, n, D, Q.dtype),), 0xff, dtype=torch.uint8, device=DEV)
    l2kv.l2kv_tree_attn(Q, K, V, ints([n]), off, n, Kt, Vt, offsets([4]), mask, O, ws)
    seen = torch.cat([torch.ones((4, n), dtype=torch.bool, device=DEV), (mask >> torch.arange(4, device=DEV)) & 1 == 1], 1)
    check(O, attend(Q, torch.cat([K[:, at:at + n], Kt], 1), torch.cat([V[:, at:at + n], Vt], 1), seen, None), n + 4)


@pytest.mark.parametrize("dtype,D", ROWS)
def test_stretches_of_the_widest_block(dtype, D):
    """Caches larger than what blocks of 64 rows are taken for."""
    new, m = [70, 40], 41_000_000 // (2 * 4 * 2 * D * (2 if dtype == torch.bfloat16 else 4))
    rows = [m, 3000]
    Q, K, V = make(D, new, rows, 16, 4, D, dtype)
    assert l2kv.l2kv_prompt_attn_workspace_bytes(2, 16, 4, 110, m, D, dtype) > 256 * 2 * 256 * D * 4
    O = run(Q, K, V, new, rows)
    verify(O, Q, K, V, new, rows)
    assert torch.equal(O, run(Q, K, V, new, rows))
    c = Case(D, new, rows, 16, 4, D, dtype)
    c.verify(c.run())


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("top,G", [(2, 4), (30, 4), (60, 4), (9, 1)])
def test_trees_over_more_than_the_caches_hold(dtype, D, top, G):
    """Bounds for which rows of the cache are read past the caches, with workgroups for each item; the same bits as with a bound for which
    they are not, where the work is cut alike."""
    nodes = [1 + (5 * s) % top for s in range(64)]
    lens = [(37 * s) % 300 for s in range(64)]
    c = Case(top + D, nodes, lens, 8 * G, 8, D, dtype)
    bound = 256_000_000 // (2 * 64 * 8 * D * (2 if dtype == torch.bfloat16 else 4)) + 1
    assert bound <= sum(c.room)
    O = c.run(bound=bound)
    c.verify(O)
    assert torch.equal(O, c.run(bound=bound - 2))


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,have", [([17000], 0), ([90] * 80, 0), ([70] * 90, 11), ([45, 80], 4000), ([5], 9000), ([100, 60], 40000)])
def test_hidden_rows_have_no_effect_however_the_work_is_cut(dtype, D, new, have):
    """The last row of every sequence, which only its last token sees, holds anything; all other tokens keep their bits."""
    rows = [n + have for n in new]
    Q, K, V = make(len(new), new, rows, 8, 2, D, dtype)
    clean = run(Q, K, V, new, rows)
    last = torch.tensor(starts(rows)[1:], device=DEV) - 1
    K[:, last], V[:, last[0::2]], V[:, last[1::2]] = float("nan"), float("inf"), float("nan")
    O = run(Q, K, V, new, rows)
    own = torch.tensor(starts(new)[1:], device=DEV) - 1
    others = torch.ones(sum(new), dtype=torch.bool, device=DEV)
    others[own] = False
    assert torch.equal(O[others], clean[others]) and not torch.isfinite(O[own]).any()


def test_another_stream():
    """Every call on a stream that is not the current one, behind work of that stream which its inputs come from."""
    from test_binding_calls_rows import CALLS
    side = torch.cuda.Stream()
    for name, (build, entry) in CALLS.items():
        a, outs = build()
        entry(**a)
        want = [a[o].clone() for o in outs]
        b, _ = build()
        inputs = {k: v for k, v in b.items() if isinstance(v, torch.Tensor) and k not in outs}
        late = {k: torch.zeros_like(v) for k, v in inputs.items()}
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
            for k, v in inputs.items():
                late[k].copy_(v)
        b.update(late)
        entry(**b, stream=side)
        side.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(b[o], w), (name, o)
