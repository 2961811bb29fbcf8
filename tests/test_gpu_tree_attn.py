"""Attention of drafted tokens over a slot cache against its definition in 64 bits."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from test_gpu_prompt_attn import DEV, ROWS, offsets, randn, starts

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def pack(seen, words):
    """[n, m] truth values -> [n, words] int32."""
    n, m = seen.shape
    bits = torch.zeros((n, words * 32), dtype=torch.int64)
    bits[:, :min(m, words * 32)] = seen[:, :words * 32].long()
    packed = (bits.view(n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)


def trees(seed, nodes):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for n in nodes:
        seen = torch.eye(n, dtype=torch.bool)
        for i in range(1, n):
            seen[i] |= seen[int(torch.randint(0, i, (1,), generator=gen))]
        out.append(seen)
    return out


class Case:
    def __init__(self, seed, nodes, lens, Hq, Hkv, D, dtype, masks=None, words=None, room=5):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.nodes, self.lens, self.room = nodes, lens, [n + room for n in lens]
        self.masks = trees(seed, nodes) if masks is None else masks
        words = max(1, (max(nodes) + 31) // 32) if words is None else words
        total, slots = sum(nodes), sum(self.room)
        self.Q = randn(gen, total, Hq, D).to(dtype)
        self.Kc = (randn(gen, Hkv, slots, D) * torch.exp(0.5 * randn(gen, Hkv, slots, 1))).to(dtype)
        self.Vc, self.Kt, self.Vt = (randn(gen, Hkv, n, D).to(dtype) for n in (slots, total, total))
        for first, n, r in zip(starts(self.room), lens, self.room):           # free slots hold anything
            self.Kc[:, first + n:first + r], self.Vc[:, first + n:first + r] = float("nan"), float("inf")
        self.mask = torch.cat([pack(m, words) for m in self.masks]).to(DEV)
        self.words = words

    def run(self, ws=None, O=None, bound=None, scale=0.0):
        total, Hq, D = self.Q.shape
        O = torch.full_like(self.Q, float("nan")) if O is None else O
        bound = max(self.lens) if bound is None else bound
        if ws is None:
            n = l2kv.l2kv_tree_attn_workspace_bytes(len(self.nodes), Hq, self.Kc.shape[0], total, bound, D, self.Q.dtype)
            ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
        l2kv.l2kv_tree_attn(self.Q, self.Kc, self.Vc, ints(self.lens), offsets(self.room), bound, self.Kt, self.Vt, offsets(self.nodes),
                            self.mask, O, ws, scale)
        return O

    def verify(self, O, scale=None):
        t, c = starts(self.nodes), starts(self.room)
        for s, (n, m) in enumerate(zip(self.nodes, self.lens)):
            if n == 0:
                continue
            here, cached = slice(t[s], t[s + 1]), slice(c[s], c[s] + m)
            K, V = torch.cat([self.Kc[:, cached], self.Kt[:, here]], 1), torch.cat([self.Vc[:, cached], self.Vt[:, here]], 1)
            own = self.masks[s].to(DEV).clone()
            own[:, self.words * 32:] = False
            seen = torch.cat([torch.ones((n, m), dtype=torch.bool, device=DEV), own], 1)
            check(O[here], attend(self.Q[here], K, V, seen, scale), n + m)


NODES = [([1], [1]), ([1, 1, 1], [0, 127, 128]), ([5, 0, 17, 8], [300, 40, 0, 64]), ([32, 33, 64], [65, 31, 500]), ([100], [1030]), ([3, 70], [0, 9])]


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("nodes,lens", NODES)
def test_trees(dtype, D, G, nodes, lens):
    case = Case(D + G, nodes, lens, 2 * G, 2, D, dtype)
    case.verify(case.run())


@pytest.mark.parametrize("G", [2, 3, 5, 6, 7, 8])
def test_groups(G):
    case = Case(G, [9, 40, 1], [200, 33, 700], 2 * G, 2, 128, torch.bfloat16)
    case.verify(case.run())


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("nodes,lens", [([6], [30000]), ([63], [17001]), ([1, 40], [9000, 20000]), ([200], [5000])])
def test_long_caches(dtype, D, nodes, lens):
    case = Case(3, nodes, lens, 4, 2, D, dtype)
    first = case.run()
    case.verify(first)
    assert torch.equal(first, case.run())


@pytest.mark.parametrize("dtype,D", ROWS)
def test_masks(dtype, D):
    """Any mask is taken as it is: rows that see nothing, themselves not, later nodes; over an empty cache such rows are zero."""
    gen = torch.Generator().manual_seed(2)
    nodes, lens = [40, 10, 35], [0, 50, 0]
    masks = [torch.rand((n, n), generator=gen) < 0.3 for n in nodes]
    masks[0][3], masks[1][2], masks[2][:] = False, False, False
    masks[2][34, 33] = True
    case = Case(1, nodes, lens, 4, 2, D, dtype, masks=masks)
    O = case.run()
    case.verify(O)
    assert (O[3] == 0).all() and (O[50:84] == 0).all() and not (O[42] == 0).any()
    assert torch.equal(O[84], case.Vt[:, 83].repeat_interleave(2, 0))


def test_more_and_fewer_mask_words_than_nodes():
    nodes, lens = [70, 20], [100, 10]
    for words in (1, 2, 3, 9):
        case = Case(4, nodes, lens, 4, 2, 128, torch.bfloat16, words=words)
        case.verify(case.run())


@pytest.mark.parametrize("dtype,D", ROWS)
def test_hidden_nodes_have_no_effect(dtype, D):
    nodes, lens = [45], [70]
    case = Case(5, nodes, lens, 4, 2, D, dtype)
    clean = case.run()
    sees = case.masks[0][:, 7]
    for bad in (float("nan"), float("inf")):
        case.Kt[:, 7], case.Vt[:, 7] = bad, bad
        got = case.run()
        assert torch.equal(got[~sees.to(DEV)], clean[~sees.to(DEV)])
        assert got[sees.to(DEV)].isnan().all()


def test_one_node_is_decode_attention():
    """One node per sequence that sees itself: the decode attention over the cache with the node's row appended."""
    lens = [513, 40, 2000]
    case = Case(6, [1, 1, 1], lens, 8, 2, 128, torch.bfloat16, room=1)
    O = case.run()
    slots = starts(case.room)
    K, V = case.Kc.clone(), case.Vc.clone()
    for s, n in enumerate(lens):
        K[:, slots[s] + n], V[:, slots[s] + n] = case.Kt[:, s], case.Vt[:, s]
    want = torch.empty((3, 8, 128), device=DEV)
    ws = torch.zeros(l2kv.l2kv_decode_ragged_workspace_bytes(3, 8, 2001, 128), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_decode_attn_ragged(case.Q, K, V, ints([n + 1 for n in lens]), offsets(case.room), 2001, want, ws)
    case.verify(O)
    # decode attention keeps its weights in fp32: off by the weights' rounding and the result's, as in attention64.allowed
    assert (O.float() - want).abs().max() <= 3 * 2.0 ** -8 * 4


def test_caches_of_a_batch():
    """[B][Hkv][T][D] caches, lengths below their rows."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    B, Hkv, T, D, lens, nodes = 2, 2, 60, 64, [60, 7], [3, 12]
    case = Case(7, nodes, lens, 4, Hkv, D, torch.float32)
    K, V = (randn(gen, B, Hkv, T, D) for _ in range(2))
    O = torch.empty_like(case.Q)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(B, 4, Hkv, 15, T, D, torch.float32), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_tree_attn(case.Q, K, V, ints(lens), torch.arange(B + 1, device=DEV) * Hkv * T, T, case.Kt, case.Vt, offsets(nodes), case.mask, O, ws)
    for s, first in enumerate(starts(case.room)[:-1]):
        case.Kc[:, first:first + lens[s]], case.Vc[:, first:first + lens[s]] = K[s, :, :lens[s]], V[s, :, :lens[s]]
    case.verify(O)


def test_nodes_behind_the_last_sequence():
    case = Case(8, [4, 6], [20, 0], 4, 2, 128, torch.bfloat16)
    want = case.run()
    O = torch.full_like(case.Q, 5.0)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(1, 4, 2, 10, 20, 128, torch.bfloat16), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_tree_attn(case.Q, case.Kc, case.Vc, ints([20]), offsets([25]), 20, case.Kt, case.Vt, offsets([4]), case.mask, O, ws)
    assert torch.equal(O[:4], want[:4]) and (O[4:] == 5.0).all()


def test_inconsistent_arrays_stay_inside():
    case = Case(9, [10, 10], [50, 50], 4, 2, 128, torch.bfloat16)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(2, 4, 2, 20, 50, 128, torch.bfloat16), dtype=torch.uint8, device=DEV)
    for off in ([0, 25, 15], [12, 5, 2], [-5, 8, 1 << 40]):
        for lens in ([50, 50], [-3, 1 << 30]):
            bad = torch.tensor(off, dtype=torch.int64, device=DEV)
            for nodes, slots in ((bad, offsets(case.room)), (offsets(case.nodes), bad * 6), (bad, bad)):
                guard = torch.full((22, 4, 128), 3.0, dtype=torch.bfloat16, device=DEV)
                l2kv.l2kv_tree_attn(case.Q, case.Kc, case.Vc, ints(lens), slots, 50, case.Kt, case.Vt, nodes, case.mask, guard[1:21], ws)
                assert (guard[0] == 3).all() and (guard[21] == 3).all()


def test_graph():
    case = Case(10, [7, 30], [4000, 90], 8, 2, 128, torch.bfloat16)
    O = torch.empty_like(case.Q)
    bound, args = 4000, (ints(case.lens), offsets(case.room))
    at = offsets(case.nodes)
    ws = torch.empty(l2kv.l2kv_tree_attn_workspace_bytes(2, 8, 2, 37, bound, 128, torch.bfloat16), dtype=torch.uint8, device=DEV)

    def call():
        l2kv.l2kv_tree_attn(case.Q, case.Kc, case.Vc, args[0], args[1], bound, case.Kt, case.Vt, at, case.mask, O, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        case.Q.copy_(randn(torch.Generator(device=DEV).manual_seed(seed), *case.Q.shape))
        O.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, case.run())
