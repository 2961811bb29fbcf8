"""Trees over caches that are read past the caches, cut into stretches that several workgroups have parts of."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend
from test_gpu_prompt_attn import DEV, ROWS, starts
from test_gpu_rows_not_finite import check_all
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("nodes,less", [([63], [500]), ([7], [0]), ([20, 9], [11, 1003])])
def test_stretches(dtype, D, nodes, less):
    """The 64-bit form, and the bits of the same call with a bound for which the rows go through the caches."""
    Hq, Hkv, n_seq = 8, 4, len(nodes)
    bound = 256_000_000 // (2 * n_seq * Hkv * D * (2 if dtype == torch.bfloat16 else 4)) + 1
    case = Case(D, nodes, [bound - x for x in less], Hq, Hkv, D, dtype, room=1100)
    assert l2kv.l2kv_tree_attn_workspace_bytes(n_seq, Hq, Hkv, sum(nodes), bound, D, dtype) > 0
    O = case.run(bound=bound)
    assert torch.equal(O, case.run(bound=bound)) and torch.equal(O, case.run(bound=bound - 2))
    t, c = starts(nodes), starts(case.room)
    for s, (n, m) in enumerate(zip(nodes, case.lens)):
        here = slice(t[s], t[s + 1])
        seen = torch.cat([torch.ones((n, m), dtype=torch.bool, device=DEV), case.masks[s].to(DEV)], 1)
        for h in range(Hkv):                                       # a KV head at a time: room for 64 bits
            q, rows = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv), slice(c[s], c[s] + m)
            K, V = torch.cat([case.Kc[h:h + 1, rows], case.Kt[h:h + 1, here]], 1), torch.cat([case.Vc[h:h + 1, rows], case.Vt[h:h + 1, here]], 1)
            check_all(O[here, q], attend(case.Q[here, q].contiguous(), K, V, seen), n + m)
