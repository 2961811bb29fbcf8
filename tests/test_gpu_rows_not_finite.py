"""NaN and infinities that a query sees, under every way the work is cut: they reach its result as they do in the definition in 64 bits, and
no other row's."""
from itertools import islice

import pytest
import torch

from attention64 import attend, check
from test_gpu_prompt_attn import DEV, make, reference, run, starts
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

NAN = float("nan")
ROWS = [(torch.bfloat16, 128), (torch.bfloat16, 256), (torch.float32, 64)]
# stretches of narrow blocks, of the widest, several items in a stretch; a workgroup for each item
CUTS = [([5], [9000]), ([37], [9000]), ([100, 60], [40100, 40060]), ([10, 1, 3], [3000, 700, 4097]), ([70] * 90, [81] * 90)]


def check_all(got, want, m):
    """As check(), and what is not finite is the same NaN or the infinity of the same sign."""
    o = want[0]
    assert torch.equal(got.isnan(), o.isnan()) and torch.equal(got.isposinf(), o.isposinf()) and torch.equal(got.isneginf(), o.isneginf())
    check(got, want, m)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", CUTS)
def test_a_query_that_is_nan(dtype, D, new, rows):
    """Every score of its row is NaN, in every part of a cut item: the row is NaN and not zeros; the rows beside it keep their bits."""
    Q, K, V = make(1, new, rows, 4, 2, D, dtype)
    clean = run(Q, K, V, new, rows)
    bad = torch.zeros(Q.shape[:2], dtype=torch.bool, device=DEV)
    bad[len(Q) // 2, 1] = bad[0, 2] = True
    Q[bad] = NAN
    got = run(Q, K, V, new, rows)
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", CUTS)
@pytest.mark.parametrize("first,count", [(0, 1), (20, 4000), (-1, 1), (-2500, 2500)])
def test_runs_of_keys_that_are_nan(dtype, D, new, rows, first, count):
    """Longer than what a workgroup takes of an item, and alone in the first or the last part: whoever sees one is NaN."""
    Q, K, V = make(2, new, rows, 4, 2, D, dtype)
    at = starts(rows)[0] + (first if first >= 0 else max(0, rows[0] + first))
    K[:, at:min(at + count, rows[0])] = NAN
    got = run(Q, K, V, new, rows)
    for where, want, m in islice(reference(Q, K, V, new, rows), 3):
        check_all(got[where], want, m)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("from_the_end", [False, True])
def test_a_run_that_ends_where_a_part_ends(dtype, D, from_the_end):
    """A part all of whose keys are NaN beside parts without any: whatever a part has, one of these runs is it."""
    new, rows = [5], [9000]
    Q, K, V = make(6, new, rows, 4, 2, D, dtype)
    Q = Q[:1].expand_as(Q).contiguous()                           # queries alike, the last of which sees every key
    for n in range(32, 1601, 32):
        K2 = K.clone()
        if from_the_end:
            K2[:, 9024 - n:] = NAN                                # whole pieces of 32 but for the last one, which has 8 rows
        else:
            K2[:, :n] = NAN
        assert run(Q, K2, V, new, rows)[-1].isnan().all(), n


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,rows", CUTS[:4])
@pytest.mark.parametrize("bad", [0.0, NAN, float("inf")])
def test_scores_of_minus_infinity(dtype, D, new, rows, bad):
    """Keys that are seen and weigh nothing: no effect, but that nothing times a value that is not finite is NaN."""
    Q, K, V = make(3, new, rows, 4, 2, D, dtype)
    Q = Q.abs() + 0.5
    top = min(rows[0], 4500)
    K[:, 100:top] = float("-inf")
    V[:, 300:top:97, 7] = bad
    got = run(Q, K, V, new, rows)
    for where, want, m in reference(Q, K, V, new, rows):
        check_all(got[where], want, m)


@pytest.mark.parametrize("dtype,D", ROWS)
def test_only_scores_of_minus_infinity(dtype, D):
    """All that a query sees weighs nothing: zeros, however the work is cut."""
    for new, rows in CUTS[:4]:
        Q, K, V = make(4, new, rows, 4, 2, D, dtype)
        Q = Q.abs() + 0.5
        K[:] = float("-inf")
        assert (run(Q, K, V, new, rows) == 0).all()


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("nodes,lens", [([6], [30000]), ([63], [40000]), ([1, 40], [9000, 20000]), ([9, 30, 2], [200, 33, 700])])
@pytest.mark.parametrize("what", ["a node's query", "cached keys", "a node's key"])
def test_trees(dtype, D, nodes, lens, what):
    case = Case(5, nodes, lens, 4, 2, D, dtype)
    if what == "a node's query":
        case.Q[0, 1] = NAN
        case.Q[-1] = NAN
    elif what == "cached keys":
        case.Kc[1, 30:lens[0] - 20] = NAN
    else:
        case.Kt[0, 0] = NAN
    got = case.run()
    t, c = starts(nodes), starts(case.room)
    for s, (n, m) in enumerate(zip(nodes, lens)):
        here, cached = slice(t[s], t[s + 1]), slice(c[s], c[s] + m)
        K, V = torch.cat([case.Kc[:, cached], case.Kt[:, here]], 1), torch.cat([case.Vc[:, cached], case.Vt[:, here]], 1)
        seen = torch.cat([torch.ones((n, m), dtype=torch.bool, device=DEV), case.masks[s].to(DEV)], 1)
        check_all(got[here], attend(case.Q[here], K, V, seen), n + m)
