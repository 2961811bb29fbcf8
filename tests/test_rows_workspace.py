"""Workspaces of prompt and tree attention over a range of sizes: no size needs more than the bound that the header gives for all of them,
and smaller calls may need more than larger ones."""
import itertools

import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding

QUERIES = [l2kv.l2kv_prompt_attn_workspace_bytes, l2kv.l2kv_tree_attn_workspace_bytes]


def compute_units():
    return l2kv.l2kv_device_info()["compute_units"] if torch.cuda.is_available() else 256


@pytest.mark.parametrize("query", QUERIES)
@pytest.mark.parametrize("dtype,D", [(binding.L2KV_BF16, 64), (binding.L2KV_BF16, 128), (binding.L2KV_BF16, 256), (binding.L2KV_F32, 64), (binding.L2KV_F32, 128)])
def test_one_bound_for_all_sizes(query, dtype, D):
    bound, sizes = compute_units() * (2048 * (D + 4) + 24), set()
    for Hkv, G in itertools.product((1, 2, 3, 8, 64), (1, 3, 4, 8)):
        if D == 256 and G > 4:
            continue
        for n_seq, total, rows in itertools.product((1, 2, 37, 1000, 1024, 1025), (1, 17, 300, 8192, 100000), (1, 333, 16384, 131072, 1 << 30)):
            sizes.add(query(n_seq, Hkv * G, Hkv, total, rows, D, dtype))
    assert max(sizes) <= bound and 0 in sizes and bound - max(sizes) < bound // 100


@pytest.mark.parametrize("query", QUERIES)
def test_it_does_not_grow_with_the_sizes(query):
    few, many = query(1, 32, 8, 300, 16384, 128, torch.bfloat16), query(1, 32, 8, 32768, 16384, 128, torch.bfloat16)
    assert few > 0 and many == 0
