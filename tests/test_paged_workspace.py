"""Workspaces of attention over pages: no size needs more than the bound that the header gives for all of them."""
import itertools

import pytest

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding
from test_rows_workspace import compute_units


@pytest.mark.parametrize("dtype,D", [(binding.L2KV_BF16, 64), (binding.L2KV_BF16, 128), (binding.L2KV_BF16, 256), (binding.L2KV_F32, 64), (binding.L2KV_F32, 128)])
def test_one_bound_for_all_sizes(dtype, D):
    bound, most = compute_units() * (2048 * (D + 4) + 24), 0
    for Hkv, G in itertools.product((1, 2, 3, 8, 64), (1, 3, 4, 8)):
        if D == 256 and G > 4:
            continue
        for n_seq, total, rows in itertools.product((1, 2, 37, 1000, 1024, 1025, 100000), (1, 17, 300, 1024, 8192, 100000), (1, 333, 16384, 131072, 1 << 30)):
            most = max(most, l2kv.l2kv_paged_attn_workspace_bytes(n_seq, Hkv * G, Hkv, total, rows, D, dtype))
    assert 0 < most <= bound
