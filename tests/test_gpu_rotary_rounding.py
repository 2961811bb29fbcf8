"""Turned elements are rounded from fp64 to fp32 and, for bf16, from there: products on and beside the middle between two numbers of either
type, at the ends of the range, and the same bits as torch's conversion."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from test_gpu_prompt_attn import DEV

pytestmark = pytest.mark.gpu

# amplitude at position 0, where an element x becomes amplitude * x exactly; what 1 becomes in bf16.  The middle between 1 and 1 + 2^-7 has the
# even neighbour below it, the next middle above it; what fp32 rounds to a middle (2^-40 away, 2^-24 away) is rounded from there.
CASES = [(1 + 2.0 ** -8 + 2.0 ** -40, 1.0), (1 + 2.0 ** -8, 1.0), (1 + 2.0 ** -8 - 2.0 ** -40, 1.0), (1 + 2.0 ** -8 + 2.0 ** -23, 1 + 2.0 ** -7),
         (1 + 3 * 2.0 ** -8 - 2.0 ** -40, 1 + 2.0 ** -6), (1 + 3 * 2.0 ** -8, 1 + 2.0 ** -6), (1 + 3 * 2.0 ** -8 - 2.0 ** -22, 1 + 2.0 ** -7),
         (1 + 2.0 ** -8 - 2.0 ** -24, 1.0), (1.25 + 2.0 ** -40, 1.25)]


def stored(x, amplitude, dtype):
    return (x.double() * amplitude).to(torch.float32).to(dtype)


@pytest.mark.parametrize("amplitude,one", CASES)
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 256), (torch.float32, 64), (torch.float32, 128)])
@pytest.mark.parametrize("layout", [0, 1])
def test_middles(amplitude, one, dtype, D, layout):
    total, Hq, Hkv = 9, 3, 2
    sign = torch.randint(0, 2, (total, Hq + 2 * Hkv, D), generator=torch.Generator().manual_seed(D)).float().mul(2).sub(1)
    scale = 2.0 ** torch.randint(-120, 120, sign.shape, generator=torch.Generator().manual_seed(1)).float()
    qkv = (sign * scale).to(dtype).to(DEV)
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    Qr = torch.empty((total, Hq, D), dtype=dtype, device=DEV)
    Kc, Vc = (torch.empty((Hkv, total, D), dtype=dtype, device=DEV) for _ in range(2))
    norms, pos = torch.empty((Hkv, total), device=DEV), torch.empty((Hkv, total), dtype=torch.int32, device=DEV)
    zero = torch.zeros(total, dtype=torch.int32, device=DEV)
    l2kv.l2kv_rotary_append(Q, K, V, zero, l2kv.l2kv_rotary_freqs(D).to(DEV), Qr, Kc, Vc, norms, pos, layout=layout, amplitude=amplitude)
    assert torch.equal(Qr, stored(Q, amplitude, dtype)) and torch.equal(Kc.transpose(0, 1), stored(K, amplitude, dtype))
    if dtype == torch.bfloat16:
        assert torch.equal(Qr, Q * one)
    assert torch.equal(Vc.transpose(0, 1), V)
    again = torch.empty_like(norms)
    l2kv.l2kv_norms(Kc, again)
    assert torch.equal(norms, again)


@pytest.mark.parametrize("amplitude", [float.fromhex("0x1.01p-130"), float.fromhex("0x1.ffp127"), float.fromhex("0x1.ffffffp127")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ends_of_the_range(amplitude, dtype):
    """Numbers below the normal ones, which have fewer bits, and infinity where the largest finite one is passed by half a step."""
    x = torch.tensor([1.0, -1.0, 0.5, 1.0625, 0.0, 1.0078125, 3.0, -2.0] * 8, device=DEV)
    K = x.to(dtype).view(1, 1, 64).contiguous()
    Kc, Vc, norms, pos = torch.empty_like(K), torch.empty_like(K), torch.empty((1, 1), device=DEV), torch.empty((1, 1), dtype=torch.int32, device=DEV)
    l2kv.l2kv_rotary_append(None, K, K, torch.zeros(1, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(64).to(DEV), None, Kc, Vc, norms, pos,
                            amplitude=amplitude)
    assert torch.equal(Kc, stored(K, amplitude, dtype))
