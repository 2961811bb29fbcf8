"""Caches [B][Hkv][T][D]: a sequence has the T rows of its head and never those of the next one, with lengths, without, and with lengths that
say more."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from paper_2406_11430_amd import binding
from test_gpu_prompt_attn import DEV, offsets, randn, starts, workspace
from test_gpu_tree_attn import ints, pack, trees

pytestmark = pytest.mark.gpu


def caches(B, Hkv, T, D, dtype):
    gen = torch.Generator(device=DEV).manual_seed(B)
    return randn(gen, B, Hkv, T, D).to(dtype), randn(gen, B, Hkv, T, D).to(dtype), torch.arange(B + 1, dtype=torch.int64, device=DEV) * Hkv * T


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("T,new", [(40, [40, 3]), (3100, [7, 30])])
@pytest.mark.parametrize("lens", [None, "more"])
def test_prompts(native, dtype, D, T, new, lens, monkeypatch):
    if not native:
        monkeypatch.setattr(binding, "_calls", binding._PythonCalls)
    B, Hkv, Hq = 2, 3, 6
    K, V, at = caches(B, Hkv, T, D, dtype)
    Q = randn(torch.Generator(device=DEV).manual_seed(9), sum(new), Hq, D).to(dtype)
    O = torch.empty_like(Q)
    lens = None if lens is None else ints([T + 1, 1 << 30])
    l2kv.l2kv_prompt_attn(Q, K, V, offsets(new), at, lens, T, O, workspace(B, Hq, Hkv, len(Q), T, D, dtype))
    for b, n in enumerate(new):
        here = slice(starts(new)[b], starts(new)[b + 1])
        seen = torch.arange(T, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + T - n
        check(O[here], attend(Q[here], K[b], V[b], seen), T)


@pytest.mark.parametrize("T", [50, 4000])
def test_trees(T):
    B, Hkv, Hq, D, nodes, dtype = 2, 2, 8, 128, [5, 9], torch.bfloat16
    K, V, at = caches(B, Hkv, T, D, dtype)
    gen = torch.Generator(device=DEV).manual_seed(3)
    Q, Kt, Vt = (randn(gen, *shape).to(dtype) for shape in ((14, Hq, D), (Hkv, 14, D), (Hkv, 14, D)))
    masks, O = trees(1, nodes), torch.empty_like(Q)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(B, Hq, Hkv, 14, T, D, dtype), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_tree_attn(Q, K, V, ints([T + 7, 2 * T]), at, T, Kt, Vt, offsets(nodes), torch.cat([pack(m, 1) for m in masks]).to(DEV), O, ws)
    for b, n in enumerate(nodes):
        here = slice(starts(nodes)[b], starts(nodes)[b + 1])
        seen = torch.cat([torch.ones((n, T), dtype=torch.bool, device=DEV), masks[b].to(DEV)], 1)
        check(O[here], attend(Q[here], torch.cat([K[b], Kt[:, here]], 1), torch.cat([V[b], Vt[:, here]], 1), seen), T + n)


def test_one_head_has_what_its_offsets_say():
    """With one KV head nothing lies behind a sequence's rows but the next sequence, and the distance of heads says nothing."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V, Q = (randn(gen, *s).bfloat16() for s in ((3, 1, 64, 128), (3, 1, 64, 128), (6, 4, 128)))
    O = torch.empty_like(Q)
    l2kv.l2kv_prompt_attn(Q, K, V, offsets([6]), torch.tensor([64, 192], device=DEV), None, 128, O, workspace(1, 4, 1, 6, 128, 128, Q.dtype))
    seen = torch.arange(128, device=DEV)[None] <= torch.arange(6, device=DEV)[:, None] + 122
    check(O, attend(Q, K.view(1, 192, 128)[:, 64:], V.view(1, 192, 128)[:, 64:], seen), 128)
