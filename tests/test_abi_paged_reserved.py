"""Refusals of l2kv_paged_append_reserved: no device is touched."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from test_abi_paged import BOTH, PAGED, PAGES_BAD
from test_abi_rows import E_ALIGN, E_NULL, E_SHAPE, ODD, P, call

RESERVED = {}
for name, value in PAGED.items():
    RESERVED[name] = value
    if name == "lens_in":
        RESERVED["ends"] = P + 128


@pytest.mark.parametrize("want,kw", BOTH + PAGES_BAD + [(E_NULL, dict(token_off=None)), (E_NULL, dict(table=None)), (E_NULL, dict(lens_in=None)),
                                                        (E_SHAPE, dict(lens_out=P)), (E_SHAPE, dict(lens_out=P + 128)), (E_ALIGN, dict(table=P + 2)),
                                                        (E_ALIGN, dict(token_off=ODD)), (E_ALIGN, dict(ends=P + 2)), (E_ALIGN, dict(ends=None, lens_in=P + 2)),
                                                        (E_SHAPE, dict(n_seq=1 << 30))])
def test_paged_append_reserved_refuses(want, kw):
    assert call("l2kv_paged_append_reserved", RESERVED, **kw) == want


def test_host_tensors_are_refused():
    Q, K = torch.zeros((3, 4, 64)), torch.zeros((2, 32, 64))
    off, n, t = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    norms, pos, freqs = K[..., 0], K[..., 0].int(), torch.zeros(16, dtype=torch.float64)
    with pytest.raises(ValueError, match="device tensors"):
        l2kv.l2kv_paged_append_reserved(Q, Q[:, :2], Q[:, :2], pos[0, :3], freqs, Q, K, K, norms, pos, off, t, 16, n, n)
