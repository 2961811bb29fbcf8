"""The accepted path of a drafted tree into the slot cache, and a whole drafted step: turned into the cache, drafted, accepted."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from test_gpu_prompt_attn import DEV, ROWS, offsets, randn, starts
from test_gpu_rotary import cache, inputs
from test_gpu_tree_attn import ints, pack, trees

pytestmark = pytest.mark.gpu


def nodes_of(seed, planes, total, D, dtype):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (randn(gen, planes, total, D).to(dtype), randn(gen, planes, total, D).to(dtype), randn(gen, planes, total),
            torch.arange(planes * total, dtype=torch.int32, device=DEV).view(planes, total))


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("planes", [1, 6])
def test_rows_and_lengths(dtype, D, planes):
    """Paths of no, one and all nodes, any order, the same node twice, outside the nodes, too long for the room; sequences without nodes."""
    nodes, have, room = [4, 9, 1, 0, 30, 2], [0, 5, 3, 2, 1, 7], [4, 3, 1, 4, 40, 0]
    path = [[0, 1, 2, 3], [8, 8, 0, 5], [7, -2, 0, 0], [0, 0, 0, 0], [29, 3, 11, 12], [0, 1, 0, 1]]
    lens = [4, 4, 3, 2, 0, 2]
    slots = [h + r for h, r in zip(have, room)]
    src, dst = nodes_of(1, planes, sum(nodes), D, dtype), cache(planes, sum(slots), D, dtype)
    want = [x.clone() for x in dst]
    out = torch.full((6,), -1, dtype=torch.int32, device=DEV)
    l2kv.l2kv_stream_append_path(*src, offsets(nodes), ints(path), ints(lens), offsets(slots), ints(have), out, *dst)
    t, c, ends = starts(nodes), starts(slots), []
    for s in range(6):
        n = 0 if nodes[s] == 0 else min(lens[s], room[s])
        ends.append(have[s] + n)
        for j in range(n):
            node = t[s] + min(max(path[s][j], 0), nodes[s] - 1)
            for w, x in zip(want, src):
                w[:, c[s] + have[s] + j] = x[:, node]
    assert out.tolist() == ends
    for x, w in zip(dst, want):
        assert torch.equal(x, w)


def test_lengths_out_of_range():
    """Path lengths below zero and above what a path has, cache lengths beyond the slots: nothing is written outside."""
    src, dst = nodes_of(2, 2, 6, 64, torch.bfloat16), cache(2, 9, 64, torch.bfloat16)
    out = torch.empty(3, dtype=torch.int32, device=DEV)
    l2kv.l2kv_stream_append_path(*src, offsets([2, 2, 2]), ints([[0, 1]] * 3), ints([-4, 100, 2]), offsets([3, 3, 3]), ints([1, 0, 7]), out, *dst)
    assert out.tolist() == [1, 2, 7]
    assert (dst[0][:, :3] == 9).all() and torch.equal(dst[0][:, 3:5], src[0][:, 2:4]) and (dst[0][:, 5:] == 9).all()


@pytest.mark.parametrize("many", [(300, 1, 1), (1, 2000, 3), (40, 5, 64)])
def test_many(many):
    n_seq, n, planes = many
    src, dst = nodes_of(3, planes, n_seq * n, 64, torch.bfloat16), cache(planes, n_seq * (n + 2), 64, torch.bfloat16)
    path = torch.randint(0, n, (n_seq, n), dtype=torch.int32, device=DEV)
    out = torch.empty(n_seq, dtype=torch.int32, device=DEV)
    l2kv.l2kv_stream_append_path(*src, offsets([n] * n_seq), path, ints([n] * n_seq), offsets([n + 2] * n_seq), ints([1] * n_seq), out, *dst)
    at = path.long() + torch.arange(n_seq, device=DEV)[:, None] * n
    for x, y in zip(dst, src):
        assert torch.equal(x.view(planes, n_seq, n + 2, *x.shape[2:])[:, :, 1:-1], y[:, at])
    assert (out == n + 1).all()


def test_a_drafted_step():
    """Prompts turned into the cache and attended to, compressed into slots, a tree drafted over them, its accepted path
    appended, the next token decoded: each step against the definition, from the step before it."""
    Hq, Hkv, D, keep = 8, 2, 128, 0.5
    new = [90, 150]
    total, dtype = sum(new), torch.bfloat16
    freqs = l2kv.l2kv_rotary_freqs(D, 500000.0).to(DEV)
    Q, K, V = inputs(1, total, Hq, Hkv, D, dtype)
    positions = torch.cat([torch.arange(n) for n in new]).to(torch.int32).to(DEV)
    Qr, (Kp, Vp, norms, pos) = torch.empty((total, Hq, D), dtype=dtype, device=DEV), cache(Hkv, total, D, dtype)
    l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, Kp, Vp, norms, pos)
    O = torch.empty_like(Qr)
    ws = torch.empty(l2kv.l2kv_prompt_attn_workspace_bytes(2, Hq, Hkv, total, 150, D, dtype), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_prompt_attn(Qr, Kp, Vp, offsets(new), offsets(new), None, 150, O, ws)
    for s, n in enumerate(new):
        here = slice(starts(new)[s], starts(new)[s + 1])
        check(O[here], attend(Qr[here], Kp[:, here], Vp[:, here], torch.ones((n, n), device=DEV).tril().bool()), n)

    kept = [l2kv.l2kv_keep_count(n, keep) for n in new]
    slots = [k + 10 for k in kept]
    idx = torch.empty((Hkv, sum(kept)), dtype=torch.int32, device=DEV)
    l2kv.l2kv_select_ragged(norms, offsets(new), offsets(kept), max(new), idx)
    Kc, Vc, norms_c, pos_c = cache(Hkv, sum(slots), D, dtype)
    l2kv.l2kv_compact_ragged(Kp, Vp, norms, idx, offsets(new), offsets(kept), max(kept), offsets(slots), Kc, Vc, norms_c, pos_c)

    nodes = [7, 12]
    tree = trees(5, nodes)
    depth = torch.cat([m.sum(1) - 1 for m in tree])
    start = torch.cat([torch.full((n,), p) for n, p in zip(nodes, new)])
    Qn, Kn, Vn = inputs(2, sum(nodes), Hq, Hkv, D, dtype)
    Qt, (Kt, Vt, norms_t, pos_t) = torch.empty((sum(nodes), Hq, D), dtype=dtype, device=DEV), cache(Hkv, sum(nodes), D, dtype)
    l2kv.l2kv_rotary_append(Qn, Kn, Vn, (start + depth).to(torch.int32).to(DEV), freqs, Qt, Kt, Vt, norms_t, pos_t)
    Ot = torch.empty_like(Qt)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(2, Hq, Hkv, sum(nodes), max(kept), D, dtype), dtype=torch.uint8, device=DEV)
    mask = torch.cat([pack(m, 1) for m in tree]).to(DEV)
    l2kv.l2kv_tree_attn(Qt, Kc, Vc, ints(kept), offsets(slots), max(kept), Kt, Vt, offsets(nodes), mask, Ot, ws)
    # accepted: from the root down to the deepest node
    paths = [m[int(m.sum(1).argmax())].nonzero().flatten().tolist() for m in tree]
    longest = max(map(len, paths))
    lens = torch.empty(2, dtype=torch.int32, device=DEV)
    l2kv.l2kv_stream_append_path(Kt, Vt, norms_t, pos_t, offsets(nodes), ints([p + [0] * (longest - len(p)) for p in paths]),
                                 ints([len(p) for p in paths]), offsets(slots), ints(kept), lens, Kc, Vc, norms_c, pos_c)
    assert lens.tolist() == [k + len(p) for k, p in zip(kept, paths)]
    for s in range(2):
        c, t, k = starts(slots)[s], starts(nodes)[s], kept[s]
        here = slice(t, t + nodes[s])
        seen = torch.cat([torch.ones((nodes[s], k), dtype=torch.bool), tree[s]], 1).to(DEV)
        check(Ot[here], attend(Qt[here], torch.cat([Kc[:, c:c + k], Kt[:, here]], 1), torch.cat([Vc[:, c:c + k], Vt[:, here]], 1), seen), k + nodes[s])
        # the accepted tokens follow the prompt, and their node saw exactly what is now in the cache
        assert (pos_c[:, c + k:c + k + len(paths[s])] == torch.arange(new[s], new[s] + len(paths[s]), device=DEV)).all()
    again = torch.empty_like(norms_c)
    l2kv.l2kv_norms(Kc, again)
    want = torch.empty((2, Hq, D), device=DEV)
    ws = torch.zeros(l2kv.l2kv_decode_ragged_workspace_bytes(2, Hq, max(slots), D), dtype=torch.uint8, device=DEV)
    last = torch.tensor([starts(nodes)[s] + paths[s][-1] for s in range(2)], device=DEV)
    l2kv.l2kv_decode_attn_ragged(Qt[last].contiguous(), Kc, Vc, lens, offsets(slots), max(slots), want, ws)
    for s in range(2):
        c, m = starts(slots)[s], int(lens[s])
        assert torch.equal(norms_c[:, c:c + m], again[:, c:c + m])
        one = attend(Qt[last[s]:last[s] + 1], Kc[:, c:c + m], Vc[:, c:c + m], torch.ones((1, m), dtype=torch.bool, device=DEV))
        check(Ot[last[s]:last[s] + 1], one, m)
        assert (want[s].double() - one[0][0]).abs().max() <= 1e-4
