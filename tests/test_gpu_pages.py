"""The pages' bookkeeping against a model that goes one entry after the other, and a serving step in pages as a whole."""
import random

import pytest
import torch

import paper_2406_11430_amd as l2kv
from attention64 import attend, check
from paged import DEV, Model, ints, pages_of, slots_of
from test_gpu_paged_append import normed, weights
from test_gpu_prompt_attn import ROWS, offsets, randn, starts
from test_gpu_rotary import close, inputs, turned

pytestmark = pytest.mark.gpu


class Pool:
    """A cache, its bookkeeping on the device and the model of it."""

    def __init__(self, n_pages, page, planes=2, D=64, dtype=torch.float32, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.page, self.n, self.model = page, n_pages, Model(n_pages, page)
        self.Kc, self.Vc = (randn(gen, planes, n_pages * page, D).to(dtype) for _ in range(2))
        self.norms, self.pos = randn(gen, planes, n_pages * page), torch.arange(planes * n_pages * page, dtype=torch.int32, device=DEV).view(planes, -1)
        self.refs, self.free, self.count = (torch.full((n,), 77, dtype=torch.int32, device=DEV) for n in (n_pages, n_pages, 1))
        self.ws = torch.full((l2kv.l2kv_pages_workspace_bytes(n_pages),), 0x5a, dtype=torch.uint8, device=DEV)

    def init(self, n_seq, width):
        t = torch.full((n_seq, width), 5, dtype=torch.int32, device=DEV)
        l2kv.l2kv_pages_init(t, self.refs, self.free, self.count)
        self.same()
        assert (t == -1).all()
        return t

    def same(self):
        assert self.refs.tolist() == self.model.refs and int(self.count) == len(self.model.free)
        assert self.free[:len(self.model.free)].tolist() == self.model.free

    def reserve(self, table, first, to, **kw):
        host, ends = table.tolist(), torch.full((len(first),), -7, dtype=torch.int32, device=DEV)
        before = [x.clone() for x in (self.Kc, self.Vc, self.norms, self.pos)]
        l2kv.l2kv_pages_reserve(table, ints(first), ints(to), ends, self.refs, self.free, self.count, self.page, self.Kc, self.Vc, self.norms, self.pos,
                                self.ws, **kw)
        want, pairs = self.model.reserve(host, first, to)
        assert ends.tolist() == want and table.tolist() == host
        self.same()
        for x in before:
            for a, b in pairs:
                x[:, b * self.page:(b + 1) * self.page] = x[:, a * self.page:(a + 1) * self.page].clone()
        for x, y in zip((self.Kc, self.Vc, self.norms, self.pos), before):
            assert torch.equal(x, y)
        return want

    def fork(self, table, lens, parents, **kw):
        out, lens_out = torch.full((len(parents), table.shape[1]), 3, dtype=torch.int32, device=DEV), ints([9] * len(parents))
        l2kv.l2kv_pages_fork(table, ints(lens), ints(parents), out, lens_out, self.refs, self.page, **kw)
        want, want_lens = self.model.fork(table.tolist(), lens, parents)
        assert out.tolist() == want and lens_out.tolist() == want_lens
        self.same()
        return out, want_lens

    def release(self, table, keep, **kw):
        host = table.tolist()
        l2kv.l2kv_pages_release(table, ints(keep), self.refs, self.free, self.count, self.page, self.ws, **kw)
        self.model.release(host, keep)
        assert table.tolist() == host
        self.same()


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("dtype,D", ROWS)
def test_branches(page, dtype, D):
    """Prompts, branches of them with the last page in common, their own copies, more pages, the end."""
    p = Pool(60, page, 3, D, dtype)
    t = p.init(3, 9)
    lens = [5 * page // 2, page, 1]
    assert p.reserve(t, [0, 0, 0], lens) == lens
    b, lens = p.fork(t, lens, [0, 2, 0, 0, 1, 7, -1])
    p.release(t, [0, 0, 0])
    more = [n + 3 for n in lens]
    assert p.reserve(b, lens, more) == more                         # the last of the three branches of the first keeps its page
    c, lens = p.fork(b, more, [1, 1, 3])
    assert p.reserve(c, lens, [n + page for n in lens]) == [n + page for n in lens]
    p.release(b, [0] * 7)
    p.release(c, [page, 0, page + 1])
    p.release(c, [0, 0, 0])
    assert int(p.count) == 60 and p.refs.sum() == 0


def test_the_same_pages_come_back():
    p = Pool(40, 16)
    t = p.init(4, 10)
    to = [33, 64, 1, 17]
    p.reserve(t, [0] * 4, to)
    first = t.clone()
    p.release(t, [0] * 4)
    p.reserve(t, [0] * 4, to)
    assert torch.equal(t, first)


def test_too_few_pages():
    """Served in order; what does not fit is left as it was, and what needs none is served, but not one that would then write a page that
    another still holds."""
    p = Pool(10, 16)
    t = p.init(4, 8)
    assert p.reserve(t, [0, 0, 0, 0], [40, 32, 33, 1]) == [40, 32, 33, 1]              # 3 + 2 + 3 + 1
    assert p.reserve(t, [40, 32, 33, 1], [41, 64, 48, 9]) == [41, 32, 48, 9]           # the second wants two and one is left
    assert p.reserve(t, [41, 32, 48, 9], [49, 33, 49, 10]) == [49, 32, 48, 10]         # one for the first, none for the others
    p.release(t, [0, 32, 0, 0])
    b, lens = p.fork(t, [0, 20, 0, 0], [1, 1, 1])
    p.release(t, [0] * 4)
    assert p.reserve(b, [20, 20, 20], [21, 21, 150]) == [21, 21, 20]                   # the third asks for more than its table has room for
    # a page of three holders that all ask; copies for the first two do not fit
    p = Pool(3, 16)
    t = p.init(1, 2)
    p.reserve(t, [0], [20])
    b, lens = p.fork(t, [20], [0, 0, 0])
    p.release(t, [0])
    assert p.reserve(b, [20] * 3, [21] * 3) == [21, 20, 20]


@pytest.mark.parametrize("first,to", [([5, -1, 0, 0], [5, 4, 129, 0]), ([9, 3, 1 << 30, -5], [2, 3, 2147483647, -1])])
def test_nothing_asked_for(first, to):
    p = Pool(10, 16)
    t = p.init(4, 8)
    assert p.reserve(t, first, to) == first and int(p.count) == 10


@pytest.mark.parametrize("n_seq,width,page", [(1, 2000, 16), (65, 40, 16), (1030, 5, 32), (2500, 3, 16), (2, 1024, 16), (1, 2049, 16), (3, 1000, 32), (8, 512, 16), (1024, 2, 16), (40, 500, 16), (3000, 11, 16), (3, 7000, 16)])
def test_many_entries(n_seq, width, page):
    """More than 1024 sequences and more entries than a pass, LDS or a workgroup takes, random lengths, forks and releases."""
    rng = random.Random(n_seq)
    n_pages = 3 * n_seq * width // 2 + 5
    p = Pool(n_pages, page, 1, 64, torch.bfloat16)
    t = p.init(n_seq, width)
    lens = [rng.randint(0, width * page * 3 // 4) for _ in range(n_seq)]
    p.reserve(t, [0] * n_seq, lens)
    b, lens = p.fork(t, lens, [rng.randrange(n_seq) for _ in range(n_seq)])
    p.release(t, [rng.choice([0, 1000000, page]) for _ in range(n_seq)])
    p.reserve(b, lens, [min(n + rng.randint(0, 2 * page), width * page) for n in lens])
    p.release(b, [rng.randint(0, width * page) for _ in range(n_seq)])
    p.release(t, [0] * n_seq), p.release(b, [0] * n_seq)
    assert int(p.count) == n_pages


def test_random_steps():
    rng = random.Random(5)
    p, lens = Pool(50, 16, 1), [0] * 6
    t = p.init(6, 12)
    for _ in range(40):
        kind = rng.choice(["grow", "grow", "branch", "cut"])
        if kind == "grow":
            lens = p.reserve(t, lens, [n + rng.choice([0, 1, 5, 40]) for n in lens])
        elif kind == "cut":
            keep = [rng.randint(0, n) for n in lens]
            p.release(t, keep)
            lens = keep
        else:
            old = t
            t, lens = p.fork(t, lens, [rng.randrange(-1, 6) for _ in range(6)])
            p.release(old, [0] * 6)


def test_inconsistent_arrays_stay_inside():
    """Counts, lists and tables of nonsense: nothing outside the arrays is written, and the calls come back."""
    for seed in range(4):
        gen = torch.Generator().manual_seed(seed)

        def nonsense(*shape):
            x = torch.randint(-2 ** 31, 2 ** 31, shape, generator=gen)
            return torch.where(torch.rand(shape, generator=gen) < 0.5, x, torch.randint(-3, 15, shape, generator=gen)).to(torch.int32).to(DEV)
        big = nonsense(400)
        guard = big.clone()
        t, refs, free, count, ends = big[10:34].view(4, 6), big[50:62], big[70:82], big[90:91], big[100:104]
        K = torch.zeros((2, 12 * 16, 64), device=DEV)
        c = (K, K.clone(), torch.zeros((2, 192), device=DEV), torch.zeros((2, 192), dtype=torch.int32, device=DEV))
        ws = torch.zeros(l2kv.l2kv_pages_workspace_bytes(12), dtype=torch.uint8, device=DEV)
        l2kv.l2kv_pages_reserve(t, nonsense(4), nonsense(4), ends, refs, free, count, 16, *c, ws)
        l2kv.l2kv_pages_release(t, nonsense(4), refs, free, count, 16, ws)
        out, lens = big[110:122].view(2, 6), big[130:132]
        l2kv.l2kv_pages_fork(t, nonsense(4), nonsense(2), out, lens, refs, 16)
        own = torch.zeros(400, dtype=torch.bool, device=DEV)
        for a, b in ((10, 34), (50, 62), (70, 82), (90, 91), (100, 104), (110, 122), (130, 132)):
            own[a:b] = True
        assert torch.equal(big[~own], guard[~own])


def test_a_graph():
    """A step of branches captured once: it leaves the pool as it found it, so every replay gives the same tables and fresh copies."""
    p = Pool(40, 16, 2)
    t, lens = p.init(3, 6), [20, 33, 48]
    p.reserve(t, [0] * 3, lens)
    b, n = torch.full_like(t, -1), ints(lens)
    parents, zero, ends, to, lens_b = ints([1, 1, 0]), ints([0] * 3), ints([0] * 3), ints([0] * 3), ints([0] * 3)

    def step():
        l2kv.l2kv_pages_release(b, zero, p.refs, p.free, p.count, 16, p.ws)
        l2kv.l2kv_pages_fork(t, n, parents, b, lens_b, p.refs, 16)
        torch.add(lens_b, 1, out=to)
        l2kv.l2kv_pages_reserve(b, lens_b, to, ends, p.refs, p.free, p.count, 16, p.Kc, p.Vc, p.norms, p.pos, p.ws)
    step()
    want = [x.clone() for x in (b, ends, lens_b, p.refs, p.count)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        p.Kc.normal_(), p.norms.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((b, ends, lens_b, p.refs, p.count), want):
            assert torch.equal(x, y)
        for s, parent in enumerate([1, 1, 0]):
            at, old = (slots_of(row, lens[parent], 16).to(DEV) for row in (b[s].tolist(), t[parent].tolist()))
            assert torch.equal(p.Kc[:, at], p.Kc[:, old]) and torch.equal(p.norms[:, at], p.norms[:, old])


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_a_step_in_pages(dtype, D):
    """Room for prompts, prompts normed and turned into it and attended to, branches, one token for each of them, attended to, compacted to half
    and the old pages given back, one more token: each step against the definition, from the step before it."""
    page, Hq, Hkv, eps = 16, 4, 2, 1e-6
    pool = Pool(80, page, Hkv, D, dtype)
    pool.Kc.fill_(float("nan")), pool.Vc.fill_(float("nan"))
    t, new = pool.init(2, 12), [90, 37]
    qw, kw = weights(1, D)
    freqs = l2kv.l2kv_rotary_freqs(D, 500000.0).to(DEV)
    cache = (pool.Kc, pool.Vc, pool.norms, pool.pos)

    def append_and_attend(seed, table, lens, new, position):
        """-> lengths behind it; checks rows, results and that what was there stayed."""
        total = sum(new)
        Q, K, V = inputs(seed, total, Hq, Hkv, D, dtype)
        positions = torch.cat([torch.arange(p, p + n) for p, n in zip(position, new)]).to(torch.int32).to(DEV)
        Qr, O = (torch.empty((total, Hq, D), dtype=dtype, device=DEV) for _ in range(2))
        out = ints([0] * len(new))
        before = [slots_of(row, n, page).to(DEV) for row, n in zip(table.tolist(), lens)]
        held = [pool.Kc[:, x].clone() for x in before]
        l2kv.l2kv_paged_append(Q, K, V, positions, freqs, Qr, *cache, offsets(new), table, page, ints(lens), out, qw, kw, eps)
        after = [a + b for a, b in zip(lens, new)]
        assert out.tolist() == after
        for x, y in zip(before, held):
            assert torch.equal(pool.Kc[:, x], y)
        ws = torch.empty(max(1, l2kv.l2kv_paged_attn_workspace_bytes(len(new), Hq, Hkv, total, max(after), D, dtype)), dtype=torch.uint8, device=DEV)
        l2kv.l2kv_paged_attn(Qr, pool.Kc, pool.Vc, offsets(new), table, page, out, max(after), O, ws)
        q = starts(new)
        want = turned(normed(K, kw, eps), positions, freqs, 0, 1.0)
        for s, (n, m) in enumerate(zip(new, after)):
            at, here = slots_of(table[s].tolist(), m, page).to(DEV), slice(q[s], q[s + 1])
            close(pool.Kc[:, at[m - n:]].transpose(0, 1), want[here])
            seen = torch.arange(m, device=DEV)[None] <= torch.arange(n, device=DEV)[:, None] + m - n
            check(O[here], attend(Qr[here], pool.Kc[:, at], pool.Vc[:, at], seen), m)
        return after

    pool.reserve_rows = lambda table, a, b: l2kv.l2kv_pages_reserve(table, ints(a), ints(b), ends, pool.refs, pool.free, pool.count, page, *cache, pool.ws)
    ends = ints([0, 0])
    pool.reserve_rows(t, [0, 0], new)
    assert ends.tolist() == new
    lens = append_and_attend(1, t, [0, 0], new, [0, 0])
    parents = [0, 1, 0]
    b, lens_b, ends = torch.full((3, 12), -1, dtype=torch.int32, device=DEV), ints([0] * 3), ints([0] * 3)
    l2kv.l2kv_pages_fork(t, ints(lens), ints(parents), b, lens_b, pool.refs, page)
    l2kv.l2kv_pages_release(t, ints([0, 0]), pool.refs, pool.free, pool.count, page, pool.ws)
    lens = [lens[x] for x in parents]
    pool.reserve_rows(b, lens, [n + 1 for n in lens])
    assert ends.tolist() == [n + 1 for n in lens]
    lens = append_and_attend(2, b, lens, [1, 1, 1], lens)
    positions = list(lens)
    keep = [l2kv.l2kv_keep_count(n, 0.5) for n in lens]
    c, lens_c = torch.full((3, 12), -1, dtype=torch.int32, device=DEV), ints([0] * 3)
    pool.reserve_rows(c, [0] * 3, keep)
    old = [slots_of(b[s].tolist(), lens[s], page).to(DEV) for s in range(3)]
    was = [x.clone() for x in cache]
    ws = torch.empty(l2kv.l2kv_paged_compress_workspace_bytes(Hkv, 3, sum(lens), sum(keep)), dtype=torch.uint8, device=DEV)
    l2kv.l2kv_paged_compress(*cache, b, ints(lens), ints(keep), c, lens_c, page, sum(lens), sum(keep), max(lens), ws)
    assert lens_c.tolist() == keep
    for s in range(3):
        at = slots_of(c[s].tolist(), keep[s], page).to(DEV)
        for h in range(Hkv):
            order = torch.sort(was[2][h, old[s]], stable=True).indices[:keep[s]].sort().values
            for x, y in zip(cache, was):
                assert torch.equal(x[h, at], y[h, old[s][order]])
    l2kv.l2kv_pages_release(b, ints([0] * 3), pool.refs, pool.free, pool.count, page, pool.ws)
    assert int(pool.count) == 80 - sum(pages_of(k, page) for k in keep)
    pool.reserve_rows(c, keep, [k + 1 for k in keep])
    append_and_attend(3, c, keep, [1, 1, 1], positions)


def test_few_pages_and_many_holders():
    """Pages run out at every place of a list of branches that share their last pages, with and without others behind them."""
    for spare in range(9):
        p = Pool(9 + spare, 16, 1)
        t = p.init(2, 8)
        p.reserve(t, [0, 0], [70, 50])
        b, lens = p.fork(t, [70, 50], [0, 0, 1, 0, 1, 1])
        if spare % 2 == 0:
            p.release(t, [0, 0])
        p.reserve(b, lens, [n + 1 for n in lens])
        p.reserve(b, lens, [n + 20 for n in lens])
