"""Attention over pages where keys and values leave the ordinary: infinities and NaN among the keys, values at the end of the range, scores that
are all minus infinity; for single tokens, which have a kernel of their own, and for chunks."""
import pytest
import torch

from attention64 import attend, check
from paged import DEV
from test_gpu_paged_attn import Case
from test_gpu_prompt_attn import ROWS

pytestmark = pytest.mark.gpu

GROUPS = [(dtype, D, G) for dtype, D in ROWS for G in (1, 4)] + [(torch.bfloat16, 128, G) for G in (6, 8)]


def held(c, s):
    return c.slots[s].to(DEV)


@pytest.mark.parametrize("dtype,D,G", GROUPS)
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("rows", [[190, 300], [9001, 40]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_keys_that_are_not_finite(dtype, D, G, new, rows, bad):
    """A NaN makes every score of its row NaN, and so every element of those who see it.  An infinity against queries of one sign is a score of
    plus infinity, and NaN as well, or of minus infinity: no weight, as if the row were not there."""
    c = Case(3, [new, new], rows, 2 * G, 2, D, dtype, 16)
    clean = c.run()
    c.Q[:new, :, 5] = c.Q[:new, :, 5].abs() + 0.5
    c.Kc[:, held(c, 0)[rows[0] // 3], 5] = bad            # seen by all queries of the first sequence
    got = c.run()
    assert torch.equal(got[new:], clean[new:])
    if bad == -float("inf"):
        at = held(c, 0)
        m = rows[0]
        seen = torch.arange(m, device=DEV)[None] <= torch.arange(new, device=DEV)[:, None] + m - new
        seen[:, m // 3] = False
        K = c.Kc[:, at].clone()
        K[:, m // 3] = 0
        check(got[:new], attend(c.Q[:new], K, c.Vc[:, at], seen), m)
    else:
        assert got[:new].isnan().all()


@pytest.mark.parametrize("dtype,D,G", GROUPS)
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("rows", [190, 5000])
def test_scores_that_are_all_minus_infinity(dtype, D, G, new, rows):
    c = Case(4, [new], [rows], 2 * G, 2, D, dtype, 32)
    c.Q[..., 7] = 1
    c.Kc[:, held(c, 0), 7] = -float("inf")
    assert (c.run() == 0).all()


@pytest.mark.parametrize("dtype,D,G", GROUPS)
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("rows,step", [(190, 0.0), (190, 0.05), (190, 3.0), (9001, 11 / 9001)])
def test_large_values(dtype, D, G, new, rows, step):
    """Weights are at most one: 190 values of 2^120, and sums of more of 2^114 whose weights fall, stay within the range."""
    c = Case(5, [new], [rows], 2 * G, 2, D, dtype, 16)
    at = held(c, 0)
    c.Q.fill_(1.0)
    c.Kc[:, at] = (torch.arange(rows, device=DEV)[:, None] * (step / D ** 0.5)).to(dtype).expand(rows, D)
    c.Vc[:, at] = c.Vc[:, at].sign() * (2.0 ** 120 if rows < 1000 else 2.0 ** 114)
    c.verify(c.run())


@pytest.mark.parametrize("dtype,D,G", GROUPS)
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("rows", [[190, 40], [7000, 700]])
def test_scores_far_apart(dtype, D, G, new, rows):
    """Scores of some thousands, of which one takes everything, wherever it is."""
    c = Case(6, [new, new], rows, 2 * G, 2, D, dtype, 64)
    c.Q *= 30
    for s, m in enumerate(rows):
        c.Kc[:, held(c, s)[m // 2]] *= 40
    c.verify(c.run())


@pytest.mark.parametrize("D,G", [(64, 1), (64, 8), (128, 4), (128, 6), (128, 8), (256, 4)])
@pytest.mark.parametrize("new,rows", [([1], [190]), ([1], [5000]), ([1] * 40, [300] * 40), ([3, 0, 0], [2000, 9, 1])])
def test_weights_of_tokens_by_themselves_are_not_rounded(D, G, new, rows):
    """No more tokens than sequences: bf16 results are off by their own rounding and by what fp32 makes of scores, exponentials and sums (the terms
    of attention64.allowed without those of the weights)."""
    c = Case(8, new, rows, 2 * G, 2, D, torch.bfloat16, 16)
    O, first = c.run().double(), 0
    for s, (n, m) in enumerate(zip(new, rows)):
        at, here = held(c, s), slice(first, first + n)
        first += n
        seen = torch.arange(m, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + m - n
        o, size, big = attend(c.Q[here], c.Kc[:, at], c.Vc[:, at], seen)
        assert ((O[here] - o).abs() <= size * (2 * (D + 4) * 2.0 ** -24 * big + (m + 8) * 2.0 ** -23) + 2.0 ** -8 * o.abs() + 1e-30).all()
