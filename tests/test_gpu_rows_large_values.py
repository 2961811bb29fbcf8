"""Values near the end of the types' range: what is summed on the way stays within it wherever the weights, which sum to one, leave the
result there, also while scores rise above the maximum that weights are relative to."""
import pytest
import torch

from test_gpu_prompt_attn import DEV, ROWS, make, run, verify
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

# Weights are at most one, so sums over 190 keys stay below 190 * 2^120 < 2^128 (and so do sums of more keys that rise: 2^120 times a
# geometric sum of at most 1 / (1 - e^-0.05) = 20.5).
LARGE = 2.0 ** 120


def rising(x, step):
    """Scores 0, step, 2 step, ... for queries of ones and the usual scale, in natural logarithms."""
    n, D = x.shape[-2:]
    return (torch.arange(n, device=DEV)[:, None] * (step / D ** 0.5) + 0 * x.float()).to(x.dtype)


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("step", [0.0, 0.05, 0.3, 3.0])
def test_prompts(dtype, D, step):
    new = rows = [190]
    Q, K, V = make(1, new, rows, 4, 2, D, dtype)
    Q, K, V = torch.ones_like(Q), rising(K, step), V.sign() * LARGE
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


@pytest.mark.parametrize("dtype,D", ROWS)
def test_keys_shared_among_workgroups(dtype, D):
    """Scores rise by 11 over 9001 keys, fewest at the top of the range."""
    new, rows = [6], [9001]
    Q, K, V = make(2, new, rows, 4, 2, D, dtype)
    Q, V = torch.ones_like(Q), V.sign() * 2.0 ** 114
    K = rising(K.new_zeros(rows[0], D), 11 / 9001).expand_as(K).contiguous()
    verify(run(Q, K, V, new, rows), Q, K, V, new, rows)


@pytest.mark.parametrize("dtype,D", ROWS)
def test_one_key_takes_everything(dtype, D):
    """A value a thousandth below the largest finite one, under a weight of nearly one, behind keys whose scores are 11 lower."""
    new = rows = [120]
    Q, K, V = make(3, new, rows, 4, 2, D, dtype)
    Q, K = torch.ones_like(Q), K * 0
    K[:, 119] = 11 / D ** 0.5
    V[:, 119] = 0.999 * torch.finfo(dtype).max
    O = run(Q, K, V, new, rows)
    assert torch.isfinite(O[:119]).all()
    # its weight is 1 / (1 + 119 e^-11) = 0.9981 or nearer to one (11 / sqrt(D) is rounded up or down by half a step)
    share = O[119].double() / V[0, 119, 0].double()
    assert (share > 0.99).all() and (share <= 1.0).all()


@pytest.mark.parametrize("dtype,D", ROWS)
def test_trees(dtype, D):
    case = Case(4, [9, 20], [100, 3000], 4, 2, D, dtype)
    case.Q.fill_(1.0)
    for first, n, m in ((0, 100, 0.05), (105, 3000, 11 / 3000)):
        case.Kc[:, first:first + n] = rising(case.Kc[:, first:first + n], m)
    case.Kt.zero_()
    case.Vc, case.Vt = torch.where(case.Vc.isfinite(), case.Vc.sign() * 2.0 ** 114, case.Vc), case.Vt.sign() * 2.0 ** 114
    case.verify(case.run())
