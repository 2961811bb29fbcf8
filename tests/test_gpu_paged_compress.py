"""Compaction of a cache in pages against a sort of the norms, exactly."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from paged import DEV, PAGES, ints, slots_of, table_of
from test_gpu_prompt_attn import ROWS, randn

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, have, keep, planes, D, dtype, page, ties=False):
        both, self.n_pages, slots = table_of(list(have) + [max(k, 0) for k in keep], page, seed)
        n = len(have)
        self.a, self.b, self.old = both[:n], both[n:], slots[:n]
        self.have, self.keep, self.page = have, keep, page
        gen = torch.Generator(device=DEV).manual_seed(seed)
        shape = (planes, self.n_pages * page)
        self.cache = [randn(gen, *shape, D).to(dtype), randn(gen, *shape, D).to(dtype),
                      torch.randint(0, 5, shape, generator=gen, device=DEV).float() if ties else torch.exp(randn(gen, *shape)),
                      torch.randint(0, 1 << 30, shape, generator=gen, device=DEV, dtype=torch.int32)]

    def run(self, total=None, kept=None, top=None, keep=None, lens=None, **kw):
        n, planes = len(self.have), self.cache[0].shape[0]
        total, kept = total or max(1, sum(self.have)), kept or max(1, sum(min(k, h) for k, h in zip(self.keep, self.have)))
        ws = torch.full((l2kv.l2kv_paged_compress_workspace_bytes(planes, n, total, kept),), 0x7f, dtype=torch.uint8, device=DEV)
        out = torch.full((n,), -9, dtype=torch.int32, device=DEV)
        self.was = [x.clone() for x in self.cache]
        l2kv.l2kv_paged_compress(*self.cache, ints(self.a), ints(lens or self.have), ints(keep or self.keep), ints(self.b), out, self.page, total, kept,
                                 top or max(1, max(self.have)), ws, **kw)
        return out.tolist()

    def verify(self, kept, have=None):
        """Every sequence keeps so many of its rows, and everything else is as it was."""
        for s, k in enumerate(kept):
            if k == 0:
                continue
            at, old = slots_of(self.b[s], k, self.page).to(DEV), self.old[s].to(DEV)
            if have is not None:
                old = old[:have[s]]
            order = torch.sort(self.was[2][:, old], dim=-1, stable=True).indices[:, :k].sort(-1).values
            for x in self.was:
                x[:, at] = x[:, old].gather(1, order if x.dim() == 2 else order[..., None].expand(-1, -1, x.shape[2]))
        for x, y in zip(self.cache, self.was):
            assert torch.equal(x, y)


# sequences of no row and one, kept whole, kept none, more asked for than there are, lengths on both sides of a page and of a workgroup's chunk
SHAPES = [([777], [389]), ([1, 0, 16, 17, 300], [1, 3, 8, 17, 1]), ([64, 65, 63, 257], [64, 99, 0, 128]), ([5] * 130, [2] * 130),
          ([3000, 2, 5000], [1500, 1, 4999])]


@pytest.mark.parametrize("have,keep", SHAPES)
@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_lengths(have, keep, dtype, D, ties, page):
    c = Case(len(have), have, keep, 3, D, dtype, page, ties)
    kept = c.run()
    assert kept == [min(k, h) for k, h in zip(keep, have)]
    c.verify(kept)


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("n_seq,most", [(1, 70000), (64, 900), (1025, 40), (3000, 9)])
def test_sizes(page, n_seq, most):
    gen = torch.Generator().manual_seed(n_seq)
    have = torch.randint(0, most + 1, (n_seq,), generator=gen).tolist()
    have[0] = most
    keep = [(h + 1) // 2 for h in have]
    c = Case(page, have, keep, 2, 64, torch.bfloat16, page)
    kept = c.run()
    assert kept == keep
    c.verify(kept)


def test_bounds():
    """Larger bounds change nothing; what goes beyond smaller ones is left out, from the last sequences on."""
    c = Case(1, [100, 50, 70], [50, 25, 35], 2, 64, torch.float32, 16)
    assert c.run(total=1000, kept=500, top=900) == [50, 25, 35]
    c.verify([50, 25, 35])
    c = Case(2, [100, 50, 70], [50, 25, 35], 2, 64, torch.float32, 16)
    assert c.run(total=120, kept=110) == [50, 20, 0]                   # twenty rows of the second are left
    c.verify([50, 20, 0], [100, 20, 0])
    c = Case(3, [100, 50, 70], [50, 25, 35], 2, 64, torch.float32, 16)
    assert c.run(kept=60, top=100) == [50, 10, 0]
    c.verify([50, 10, 0])
    c = Case(4, [100, 50, 70], [50, 25, 35], 2, 64, torch.float32, 16)
    assert c.run(top=60) == [50, 25, 35]
    c.verify([50, 25, 35], [60, 50, 60])


def test_room_of_the_new_pages():
    """As many rows as the new table has room for; a row whose entry is no page is not written; negative numbers keep nothing."""
    c = Case(5, [100, 50, 40], [50, 25, 10], 2, 128, torch.bfloat16, 16)
    c.b = [row[:2] for row in c.b]
    c.b[1][1] = -1
    kept = c.run(keep=[50, 25, -4])
    assert kept == [32, 25, 0]
    c.b[1][1] = c.n_pages                                              # a page that is not there, for the rows of it
    for x in range(4):
        c.was[x] = torch.cat([c.was[x], torch.zeros_like(c.was[x][:, :16])], 1)
    c.cache = [torch.cat([x, torch.zeros_like(x[:, :16])], 1) for x in c.cache]
    old = [x.clone() for x in c.was]
    for s, k in ((0, 32), (1, 16)):
        at, src = slots_of(c.b[s], k, 16).to(DEV), c.old[s].to(DEV)
        all_kept = torch.sort(old[2][:, src], dim=-1, stable=True).indices[:, :kept[s]].sort(-1).values[:, :k]
        for x in c.was:
            x[:, at] = x[:, src].gather(1, all_kept if x.dim() == 2 else all_kept[..., None].expand(-1, -1, x.shape[2]))
    for x, y in zip(c.cache, c.was):
        assert torch.equal(x, y)


def test_shared_rows_and_a_graph():
    """Two sequences with the same pages keep different numbers of rows; captured, and replayed with other norms and counts."""
    c = Case(6, [90, 90], [45, 20], 2, 64, torch.bfloat16, 32)
    c.a[1] = c.a[0]
    c.old[1] = c.old[0]
    assert c.run() == [45, 20]
    c.verify([45, 20])
    ws = torch.empty(l2kv.l2kv_paged_compress_workspace_bytes(2, 2, 180, 65), dtype=torch.uint8, device=DEV)
    a, b, lens, keep, out = ints(c.a), ints(c.b), ints([90, 90]), ints([45, 20]), ints([0, 0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2kv.l2kv_paged_compress(*c.cache, a, lens, keep, b, out, 32, 180, 65, 90, ws)
    for counts in ([45, 20], [10, 12], [1, 20]):
        c.cache[2].normal_().abs_(), c.cache[0].normal_()
        keep.copy_(ints(counts))
        c.was = [x.clone() for x in c.cache]
        graph.replay()
        torch.cuda.synchronize()
        assert out.tolist() == counts
        c.verify(counts)


def test_norms_that_are_not_finite():
    c = Case(7, [200], [100], 2, 64, torch.float32, 16)
    slots = c.old[0].to(DEV)
    c.cache[2][:, slots[::3]] = float("inf")
    assert c.run() == [100]
    c.verify([100])


@pytest.mark.parametrize("have", [[1024, 3], [1025, 7], [2048, 2049], [4100], [8192, 8193], [16385, 30000], [32768, 1], [32769, 500]])
@pytest.mark.parametrize("ties", [False, True])
def test_long_sequences(have, ties):
    """Every number of keys that a lane of the selection holds, and sequences that it does not hold."""
    keep = [h // 3 + 1 for h in have]
    c = Case(sum(have), have, keep, 2, 64, torch.bfloat16, 64, ties)
    assert c.run() == keep
    c.verify(keep)


@pytest.mark.parametrize("have,keep", [([40000], [20001]), ([131072], [13107]), ([100003], [100003]), ([100003], [1]), ([33000, 0, 500, 40000, 65536], [100, 3, 500, 0, 40000])])
@pytest.mark.parametrize("planes", [1, 3, 17])
@pytest.mark.parametrize("ties", [False, True])
def test_few_and_long_sequences(have, keep, planes, ties):
    """Sequences that several workgroups select from, empty ones and short ones among them; with too many planes one each."""
    c = Case(len(have) + planes, have, keep, planes, 64, torch.bfloat16, 16, ties)
    kept = [min(k, h) for k, h in zip(keep, have)]
    assert c.run() == kept
    c.verify(kept)


def test_bounds_of_long_sequences():
    have, keep = [50000, 40000, 70000], [25000, 20000, 35000]
    for bounds, kept, seen in ((dict(total=400000, kept=100000, top=300000), keep, have), (dict(total=95000, kept=60000, top=90000), [25000, 20000, 5000], [50000, 40000, 5000]),
                               (dict(total=52000, top=50000), [25000, 2000, 0], [50000, 2000, 0]), (dict(kept=30000, top=70000), [25000, 5000, 0], have),
                               (dict(top=45000), keep, [45000, 40000, 45000])):
        c = Case(1, have, keep, 2, 64, torch.bfloat16, 16)
        assert c.run(**bounds) == kept
        c.verify(kept, seen)


def test_the_least_workspace_and_one_of_more_planes():
    """A workspace of a call with more planes is enough; the selection is the same."""
    have, keep, planes = [90000], [30000], 2
    c = Case(2, have, keep, planes, 64, torch.bfloat16, 16)
    ws = torch.empty(l2kv.l2kv_paged_compress_workspace_bytes(65, 1, 90000, 30000) * planes // 65 + 64, dtype=torch.uint8, device=DEV)
    assert len(ws) < l2kv.l2kv_paged_compress_workspace_bytes(planes, 1, 90000, 30000)
    out = ints([0])
    c.was = [x.clone() for x in c.cache]
    l2kv.l2kv_paged_compress(*c.cache, ints(c.a), ints(have), ints(keep), ints(c.b), out, 16, 90000, 30000, 90000, ws)
    assert out.tolist() == keep
    c.verify(keep)


def test_a_graph_of_long_sequences():
    c = Case(3, [60000, 50000], [30000, 25000], 2, 64, torch.bfloat16, 32)
    ws = torch.empty(l2kv.l2kv_paged_compress_workspace_bytes(2, 2, 110000, 55000), dtype=torch.uint8, device=DEV)
    a, b, lens, keep, out = ints(c.a), ints(c.b), ints([60000, 50000]), ints([30000, 25000]), ints([0, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2kv.l2kv_paged_compress(*c.cache, a, lens, keep, b, out, 32, 110000, 55000, 60000, ws)
    for counts, rows in (([30000, 25000], [60000, 50000]), ([0, 20000], [5, 45000]), ([29999, 1], [60000, 1])):
        c.cache[2].normal_().abs_(), c.cache[0].normal_()
        keep.copy_(ints(counts)), lens.copy_(ints(rows))
        c.was = [x.clone() for x in c.cache]
        graph.replay()
        torch.cuda.synchronize()
        assert out.tolist() == counts
        c.verify(counts, rows)


@pytest.mark.parametrize("have,keep,planes", [([8192], [8192], 1), ([8193], [8192], 1), ([8192, 8192, 7], [1, 8192, 3], 2), ([4096], [4096], 200), ([30] * 256, [29] * 256, 1),
                                              ([30] * 257, [29] * 257, 1), ([40, 0, 4000] * 20, [40, 5, 2000] * 20, 2), ([1], [1], 1)])
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 128)])
def test_shares_of_short_sequences(have, keep, planes, dtype, D):
    """The largest sequences, and the most of them, that are selected from and copied in one launch, and the next larger."""
    c = Case(len(have), have, keep, planes, D, dtype, 16)
    kept = [min(k, h) for k, h in zip(keep, have)]
    assert c.run() == kept
    c.verify(kept)


@pytest.mark.parametrize("have,planes", [([900], 300), ([2000, 3], 150), ([4000], 260), ([8000], 130), ([20000, 9000], 20), ([16000], 33), ([32768], 33), ([32768], 32), ([16001], 32)])
@pytest.mark.parametrize("ties", [False, True])
def test_many_planes(have, planes, ties):
    """As many heads as the selection and the copy go apart for, at every number of keys of a lane, and the most that go together."""
    keep = [h // 10 for h in have]
    c = Case(planes, have, keep, planes, 64, torch.bfloat16, 16, ties)
    assert c.run() == keep
    c.verify(keep)


def test_uneven_batches():
    """One long sequence among short ones, kept alike and not."""
    for keep in ([1400, 3, 10, 0, 200], [4800, 1, 30, 9, 1], [1, 11, 30, 9, 650]):
        c = Case(sum(keep), [4827, 11, 30, 9, 650], keep, 20, 128, torch.bfloat16, 64)
        assert c.run() == keep
        c.verify(keep)
