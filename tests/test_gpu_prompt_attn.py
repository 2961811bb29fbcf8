"""Causal attention of packed prompts against its definition in 64 bits."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.bfloat16, 256), (torch.float32, 128), (torch.float32, 64)]


def starts(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return out


def offsets(lens):
    return torch.tensor(starts(lens), dtype=torch.int64, device=DEV)


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def make(seed, new, rows, Hq, Hkv, D, dtype, spread=0.5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    Q = randn(gen, sum(new), Hq, D)
    K = randn(gen, Hkv, sum(rows), D) * torch.exp(spread * randn(gen, Hkv, sum(rows), 1))
    return Q.to(dtype), K.to(dtype), randn(gen, Hkv, sum(rows), D).to(dtype)


def workspace(n_seq, Hq, Hkv, total_q, max_kv, D, dtype):
    n = l2kv.l2kv_prompt_attn_workspace_bytes(n_seq, Hq, Hkv, total_q, max_kv, D, dtype)
    return torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)          # NaN wherever it is read before it is written


def run(Q, K, V, new, rows, scale=0.0, ws=None, O=None, **kw):
    Hkv = K.shape[0]
    O = torch.full(Q.shape, float("nan"), dtype=Q.dtype, device=DEV) if O is None else O
    top = max(1, max(rows))
    ws = workspace(len(new), Q.shape[1], Hkv, Q.shape[0], top, Q.shape[2], Q.dtype) if ws is None else ws
    l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), offsets(rows), None, top, O, ws, scale, **kw)
    return O


def reference(Q, K, V, new, rows, scale=None, keep=None):
    q, k = starts(new), starts(rows)
    for s, (n, m) in enumerate(zip(new, rows)):
        i = torch.arange(n, device=DEV)[:, None]
        seen = torch.arange(m, device=DEV)[None] <= i + m - n
        yield slice(q[s], q[s + 1]), attend(Q[q[s]:q[s + 1]], K[:, k[s]:k[s + 1]], V[:, k[s]:k[s + 1]], seen, scale), m


def verify(O, *args, **kw):
    for where, want, m in reference(*args, **kw):
        check(O[where], want, m)


# lengths on both sides of a tile of 32 keys, of 64 and of 128, of a block of rows; empty sequences; more rows than queries and fewer
LENGTHS = [([1], [1]), ([2, 1, 33], [2, 1, 33]), ([31, 32, 33, 0, 64, 65], [31, 32, 33, 0, 64, 65]), ([127, 128, 129], [127, 128, 129]),
           ([5, 1, 40], [300, 257, 40]), ([70, 3, 9, 4], [20, 1, 0, 133]), ([1, 1, 1, 1], [511, 512, 513, 0])]


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("G", [1, 3, 4])
@pytest.mark.parametrize("new,rows", LENGTHS)
def test_lengths(dtype, D, G, new, rows):
    Hkv = 2
    Q, K, V = make(len(new) + D, new, rows, Hkv * G, Hkv, D, dtype)
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


@pytest.mark.parametrize("G", [2, 5, 6, 7, 8])
@pytest.mark.parametrize("new,rows", [([1, 7], [90, 7]), ([200, 61], [200, 700])])
def test_groups(G, new, rows):
    Q, K, V = make(G, new, rows, 3 * G, 3, 128, torch.bfloat16)
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", [([1], [20011]), ([3, 2], [9000, 4097]), ([150], [9001]), ([700], [700])])
def test_keys_shared_among_workgroups(dtype, D, new, rows):
    Q, K, V = make(7, new, rows, 4, 2, D, dtype)
    assert l2kv.l2kv_prompt_attn_workspace_bytes(len(new), 4, 2, sum(new), max(rows), D, dtype) > 0
    first = run(Q, K, V, new, rows)
    verify(first, Q, K, V, new, rows)
    assert torch.equal(first, run(Q, K, V, new, rows))


@pytest.mark.parametrize("dtype,D", ROWS)
def test_many_blocks(dtype, D):
    new = [1500, 0, 777, 2, 1]
    Q, K, V = make(3, new, new, 16, 8, D, dtype)
    verify(run(Q, K, V, new, new), Q, K, V, new, new)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("kind", ["rising", "steep", "flat", "one key"])
def test_scores(dtype, D, kind):
    """The running maximum moves in every tile, by more and by less than what is let pass; one key takes everything."""
    new = rows = [190]
    Q, K, V = make(11, new, rows, 4, 2, D, dtype)
    if kind == "one key":
        K[:, 77] = Q[100, 0] * 4
    elif kind == "flat":
        K.zero_()
    else:
        step = 0.05 if kind == "rising" else 3.0
        Q = (Q * 0 + 1).to(dtype)
        K = (torch.arange(190, device=DEV)[None, :, None] * (step / D ** 0.5) + 0 * K.float()).to(dtype)
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


def test_scale():
    new = rows = [45]
    Q, K, V = make(2, new, rows, 2, 2, 64, torch.float32)
    verify(run(Q, K, V, new, rows, scale=0.7), Q, K, V, new, rows, scale=0.7)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_query_does_not_see_has_no_effect(dtype, D, bad):
    """Rows behind a query, behind the sequence and beside it hold infinities and NaN, in values and in keys."""
    new, rows = [100, 20], [140, 20]
    Q, K, V = make(5, new, rows, 4, 2, D, dtype)
    K2, V2 = K.clone(), V.clone()
    K2[:, 138:140], V2[:, 137:140] = bad, bad                     # seen by the last three queries of the first sequence only
    V2[:, 60, 5] = bad                                            # seen by queries from 20 on, in one column
    K2[:, 159], V2[:, 159] = bad, bad                             # by the last query of the second
    got, clean = run(Q, K2, V2, new, rows), run(Q, K, V, new, rows)
    before = list(range(0, 20)) + list(range(100, 119))
    assert torch.equal(got[before], clean[before])
    columns = [d for d in range(D) if d != 5]
    assert torch.equal(got[20:97][..., columns], clean[20:97][..., columns])
    if bad != bad:
        assert got[20:97, :, 5].isnan().all() and got[97:100].isnan().all() and got[119].isnan().all()
    else:
        assert (got[20:97, :, 5] == bad).all()


def test_what_lies_outside_the_sequences():
    """Rows between and behind the sequences hold NaN, tokens behind the last sequence keep their output, and a sequence may be read from
    a cache [B][Hkv][T][D] with lengths of its own."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    B, Hkv, T, D, Hq = 3, 2, 80, 128, 8
    lens, new = [80, 33, 0], [4, 33, 2]
    K, V = (randn(gen, B, Hkv, T, D).bfloat16() for _ in range(2))
    for b, n in enumerate(lens):
        K[b, :, n:], V[b, :, n:] = float("nan"), float("nan")
    Q = randn(gen, sum(new) + 5, Hq, D).bfloat16()
    O = torch.full_like(Q, 7.0)
    ws = workspace(B, Hq, Hkv, len(Q), T, D, torch.bfloat16)
    at = torch.arange(B + 1, dtype=torch.int64, device=DEV) * Hkv * T
    l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), at, torch.tensor(lens, dtype=torch.int32, device=DEV), T, O, ws)
    assert (O[sum(new):] == 7.0).all()
    q = starts(new)
    for b, (n, m) in enumerate(zip(new, lens)):
        seen = torch.arange(m, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + m - n
        check(O[q[b]:q[b + 1]], attend(Q[q[b]:q[b + 1]], K[b, :, :m], V[b, :, :m], seen), m)
    assert (O[q[2]:q[3]] == 0).all()


def test_queries_of_a_projection():
    gen = torch.Generator(device=DEV).manual_seed(4)
    new = rows = [50, 3]
    both = randn(gen, 53, 12, 64)
    _, K, V = make(4, new, rows, 4, 4, 64, torch.float32)
    Q = both[:, 4:8]
    verify(run(Q, K, V, new, rows, O=torch.empty(53, 4, 64, device=DEV)), Q.contiguous(), K, V, new, rows)


def test_far_offsets():
    """Rows whose place passes 32 bits, in elements and in bytes."""
    D, rows = 128, (1 << 24) + 5000
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V = (torch.empty((1, rows, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    first = rows - 300
    K[:, first:], V[:, first:] = randn(gen, 1, 300, D).bfloat16(), randn(gen, 1, 300, D).bfloat16()
    Q = randn(gen, 20, 2, D).bfloat16()
    O = torch.empty_like(Q)
    ws = workspace(1, 2, 1, 20, 300, D, torch.bfloat16)
    l2kv.l2kv_prompt_attn(Q, K, V, offsets([20]), torch.tensor([first, rows], dtype=torch.int64, device=DEV), None, 300, O, ws)
    verify(O, Q, K[:, first:], V[:, first:], [20], [300])


def test_inconsistent_offsets_stay_inside():
    """Offsets that fall, run past the end or are negative: meaningless results, but nothing outside the tensors."""
    new = rows = [40, 40]
    Q, K, V = make(6, new, rows, 4, 2, 128, torch.bfloat16)
    ws = workspace(2, 4, 2, 80, 80, 128, torch.bfloat16)
    for off in ([0, 90, 70], [50, 20, 10], [-5, 30, 1 << 40], [0, 0, 0]):
        bad = torch.tensor(off, dtype=torch.int64, device=DEV)
        for q, k in ((bad, offsets(rows)), (offsets(new), bad), (bad, bad)):
            guard = torch.full((82, 4, 128), 3.0, dtype=torch.bfloat16, device=DEV)
            l2kv.l2kv_prompt_attn(Q, K, V, q, k, None, 80, guard[1:81], ws)
            assert (guard[0] == 3).all() and (guard[81] == 3).all()


def test_lengths_beyond_the_bound():
    """max_kv sizes the cut only: rows beyond it are attended to."""
    new, rows = [3, 200], [5000, 900]
    Q, K, V = make(8, new, rows, 4, 2, 128, torch.bfloat16)
    O = torch.empty_like(Q)
    for bound in (1, 600, 2000):
        l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), offsets(rows), None, bound, O, workspace(2, 4, 2, 203, bound, 128, torch.bfloat16))
        verify(O, Q, K, V, new, rows)


def test_streams_and_graphs():
    """A call on another stream, and two graphs that share a workspace, replayed in turn on fresh inputs."""
    shapes = [([2, 5], [3000, 60]), ([300], [300])]
    ws = torch.zeros(max(l2kv.l2kv_prompt_attn_workspace_bytes(len(n), 4, 2, sum(n), max(r), 128, torch.bfloat16) for n, r in shapes),
                     dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    held = []
    for new, rows in shapes:
        Q, K, V = make(1, new, rows, 4, 2, 128, torch.bfloat16)
        O, q, k = torch.empty_like(Q), offsets(new), offsets(rows)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            l2kv.l2kv_prompt_attn(Q, K, V, q, k, None, max(rows), O, ws)
        torch.cuda.current_stream().wait_stream(side)
        verify(O, Q, K, V, new, rows)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            l2kv.l2kv_prompt_attn(Q, K, V, q, k, None, max(rows), O, ws)
        held.append((graph, Q, K, V, O, new, rows, q, k))
    for round_ in range(3):
        for graph, Q, K, V, O, new, rows, q, k in held:
            for t, fresh in zip((Q, K, V), make(50 + round_, new, rows, 4, 2, 128, torch.bfloat16)):
                t.copy_(fresh)
            O.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(O, run(Q, K, V, new, rows))
