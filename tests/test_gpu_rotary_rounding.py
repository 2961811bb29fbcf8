"""Turned elements are rounded once: products just above and just below the middle between two bf16 numbers, where a rounding to fp32 on the
way lands on the middle itself."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from test_gpu_prompt_attn import DEV

pytestmark = pytest.mark.gpu

# amplitude at position 0, where an element x becomes amplitude * x exactly, and that number rounded to bf16 (8 bits): the middle between
# 1 and 1 + 2^-7 has the even neighbour below it, the next middle above it.  Last: a middle of fp32 as well, and no middle at all.
CASES = [(1 + 2.0 ** -8 + 2.0 ** -40, 1 + 2.0 ** -7), (1 + 2.0 ** -8, 1.0), (1 + 2.0 ** -8 - 2.0 ** -40, 1.0),
         (1 + 3 * 2.0 ** -8 - 2.0 ** -40, 1 + 2.0 ** -7), (1 + 3 * 2.0 ** -8, 1 + 2.0 ** -6), (1 + 3 * 2.0 ** -8 + 2.0 ** -40, 1 + 2.0 ** -6),
         (1 + 2.0 ** -8 + 2.0 ** -24, 1 + 2.0 ** -7), (1 + 2.0 ** -8 - 2.0 ** -24, 1.0), (1.25 + 2.0 ** -40, 1.25)]


@pytest.mark.parametrize("amplitude,want", CASES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("layout", [0, 1])
def test_once(amplitude, want, D, layout):
    total, Hq, Hkv = 9, 3, 2
    sign = torch.randint(0, 2, (total, Hq + 2 * Hkv, D), generator=torch.Generator().manual_seed(D)).float().mul(2).sub(1)
    scale = 2.0 ** torch.randint(-120, 120, sign.shape, generator=torch.Generator().manual_seed(1)).float()
    qkv = (sign * scale).to(torch.bfloat16).to(DEV)
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    Qr = torch.empty((total, Hq, D), dtype=torch.bfloat16, device=DEV)
    Kc, Vc = (torch.empty((Hkv, total, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    norms, pos = torch.empty((Hkv, total), device=DEV), torch.empty((Hkv, total), dtype=torch.int32, device=DEV)
    zero = torch.zeros(total, dtype=torch.int32, device=DEV)
    l2kv.l2kv_rotary_append(Q, K, V, zero, l2kv.l2kv_rotary_freqs(D).to(DEV), Qr, Kc, Vc, norms, pos, layout=layout, amplitude=amplitude)
    assert torch.equal(Qr, Q * want) and torch.equal(Kc.transpose(0, 1), K * want) and torch.equal(Vc.transpose(0, 1), V)
    again = torch.empty_like(norms)
    l2kv.l2kv_norms(Kc, again)
    assert torch.equal(norms, again)


@pytest.mark.parametrize("amplitude", [float.fromhex("0x1.01p-130"), float.fromhex("0x1.ffp127")])
def test_ends_of_the_range(amplitude):
    """Numbers below the normal ones, which have fewer bits, and infinity where the largest finite one is passed by half a step."""
    x = torch.tensor([1.0, -1.0, 0.5, 1.0625, 0.0, 1.0078125, 3.0, -2.0] * 8, device=DEV)
    K = x.to(torch.bfloat16).view(1, 1, 64).contiguous()
    Kc, Vc, norms, pos = torch.empty_like(K), torch.empty_like(K), torch.empty((1, 1), device=DEV), torch.empty((1, 1), dtype=torch.int32, device=DEV)
    l2kv.l2kv_rotary_append(None, K, K, torch.zeros(1, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(64).to(DEV), None, Kc, Vc, norms, pos,
                            amplitude=amplitude)
    exact = x.double() * amplitude
    step = torch.clamp(torch.exp2(torch.floor(torch.log2(exact.abs().clamp(min=2.0 ** -140))) - 7), min=2.0 ** -133)
    rounded = torch.round(exact / step) * step                            # to the even neighbour
    assert torch.equal(Kc.view(-1).double(), torch.where(rounded.abs() < 2.0 ** 128, rounded, torch.copysign(torch.full_like(rounded, float("inf")), rounded)))
