"""Compaction in pages orders rows by the bits of their norms, infinities and NaN of any kind among them, in every way that it selects."""
import pytest
import torch

from paged import DEV
from test_gpu_paged_compress import Case

pytestmark = pytest.mark.gpu

INF = 0x7f800000
# infinity, the first NaN behind it, the usual one, the last; the same with the sign's bit, which are larger still
BITS = [INF, INF + 1, 0x7fc00000, 0x7fffffff, INF + (1 << 31), 0xffc00000, 0xffffffff]
# (rows, planes): one launch with the copy; norms in registers; by several workgroups; gathered first, one workgroup each
WAYS = [([200, 64], 2), ([30000, 777], 40), ([40000, 1, 33000], 2), ([33000], 70), ([20] * 1100, 1)]


def select(bits, k):
    """Rows with the k lowest bits, among equals the lower ones, ascending."""
    return torch.sort(bits.long() & 0xffffffff, dim=-1, stable=True).indices[..., :k].sort(-1).values


@pytest.mark.parametrize("have,planes", WAYS)
@pytest.mark.parametrize("finite,kept", [(0.6, 0.5), (0.6, 0.75), (0.6, 1.0), (0.0, 0.4), (0.99, 0.995)])
def test_norms_that_are_not_finite(have, planes, finite, kept):
    keep = [max(1, round(h * kept)) for h in have]
    c = Case(len(have) + planes, have, keep, planes, 64, torch.bfloat16, 16)
    gen = torch.Generator(device=DEV).manual_seed(7)
    shape = c.cache[2].shape
    bad = torch.tensor([b - (1 << 32) if b >> 31 else b for b in BITS], dtype=torch.int32, device=DEV)
    bits = torch.where(torch.rand(shape, generator=gen, device=DEV) < finite, c.cache[2].view(torch.int32),
                       bad[torch.randint(0, len(BITS), shape, generator=gen, device=DEV)])
    c.cache[2] = bits.view(torch.float32)
    assert c.run() == keep
    was, got = ([x.view(torch.int32) if x.dtype == torch.float32 else x for x in cache] for cache in (c.was, c.cache))
    most, seqs = max(have), torch.arange(len(have), device=DEV)
    slots = torch.zeros((len(have), most), dtype=torch.int64, device=DEV)
    for s, x in enumerate(c.old):
        slots[s, :have[s]] = x.to(DEV)
    to = torch.tensor([[e * 16 + i for e in row for i in range(16)][:max(keep)] + [-1] * (max(keep) - 16 * len(row)) for row in c.b], device=DEV)
    for s in seqs.tolist():
        at, old = to[s, :keep[s]], slots[s, :have[s]]
        rows = select(was[2][:, old], keep[s])
        for x in was:
            x[:, at] = x[:, old].gather(1, rows if x.dim() == 2 else rows[..., None].expand(-1, -1, x.shape[2]))
    for x, y in zip(got, was):
        assert torch.equal(x, y)
