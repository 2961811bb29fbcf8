"""Rotary positions on the way into the cache against their definition in 64 bits."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding
from attention64 import HALF_STEP
from test_gpu_prompt_attn import DEV, ROWS, offsets, randn, starts

pytestmark = pytest.mark.gpu


def turned(x, positions, freqs, interleaved, amplitude):
    R = 2 * len(freqs)
    i = torch.arange(R // 2, device=DEV)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    angle = positions.double()[:, None] * freqs[None]
    c, s = torch.cos(angle)[:, None] * amplitude, torch.sin(angle)[:, None] * amplitude
    y = x.double()
    x1, x2 = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def close(got, want, far=0.0):
    """One rounding of the result (half a step of it), and the angle's error, in 64 bits, on rows of a few units."""
    assert ((got.double() - want).abs() <= HALF_STEP[got.dtype] * want.abs() * (1 + 2.0 ** -10) + 1e-9 + far).all()


def inputs(seed, total, Hq, Hkv, D, dtype):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    qkv = randn(gen, total, Hq + 2 * Hkv, D).to(dtype)
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]


def cache(Hkv, slots, D, dtype):
    K, V = (torch.full((Hkv, slots, D), 9.0, dtype=dtype, device=DEV) for _ in range(2))
    return K, V, torch.full((Hkv, slots), 9.0, device=DEV), torch.full((Hkv, slots), 9, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype,D,rot", [(*row, rot) for row in ROWS for rot in (16, 48, 64, 128, 256) if rot <= row[1]])
@pytest.mark.parametrize("layout", [0, 1])
def test_prompts(dtype, D, layout, rot):
    """Packed, straight from a projection, part of the head and all of it, near and far positions of both signs."""
    total, Hq, Hkv = 133, 6, 2
    Q, K, V = inputs(rot, total, Hq, Hkv, D, dtype)
    positions = torch.cat([torch.arange(100), torch.arange(33) * 31251 - 1000]).to(torch.int32).to(DEV)
    freqs = l2kv.l2kv_rotary_freqs(rot, 10000.0).to(DEV)
    Qr = torch.empty((total, Hq, D), dtype=dtype, device=DEV)
    Kc, Vc, norms, pos = cache(Hkv, total, D, dtype)
    l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, Kc, Vc, norms, pos, layout=layout, amplitude=1.25)
    close(Qr, turned(Q, positions, freqs, layout, 1.25))
    close(Kc.transpose(0, 1), turned(K, positions, freqs, layout, 1.25))
    assert torch.equal(Vc, V.transpose(0, 1)) and torch.equal(Qr[..., rot:], Q[..., rot:])
    assert torch.equal(pos, positions.expand(Hkv, total))
    again = torch.empty_like(norms)
    l2kv.l2kv_norms(Kc, again)
    assert torch.equal(norms, again)                              # bit for bit the norms of the rows as stored


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("new,have,room", [([1, 1, 1], [0, 7, 20], [4, 4, 4]), ([3, 0, 70, 2, 1], [2, 5, 0, 9, 4], [2, 2, 3, 1, 0]),
                                           ([1] * 200, list(range(200)), [1] * 200)])
def test_slots(dtype, D, new, have, room):
    """Behind the occupied slots of every sequence; what finds no room is not stored; everything else stays as it was."""
    total, Hq, Hkv = sum(new), 2, 2
    slots = [h + r for h, r in zip(have, room)]
    Q, K, V = inputs(len(new), total + 2, Hq, Hkv, D, dtype)       # two tokens that no sequence has
    positions = (torch.arange(total + 2, dtype=torch.int32) * 3).to(DEV)
    freqs = l2kv.l2kv_rotary_freqs(D, 500000.0, binding.L2KV_ROTARY_LINEAR, 4.0).to(DEV)
    Qr = torch.full((total + 2, Hq, D), 9.0, dtype=dtype, device=DEV)
    Kc, Vc, norms, pos = cache(Hkv, sum(slots), D, dtype)
    lens_in = torch.tensor(have, dtype=torch.int32, device=DEV)
    lens_out = torch.full_like(lens_in, -1)
    l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, Kc, Vc, norms, pos, offsets(new), offsets(slots), lens_in, lens_out)
    assert lens_out.tolist() == [h + min(n, r) for n, h, r in zip(new, have, room)]
    close(Qr[:total], turned(Q, positions, freqs, 0, 1.0)[:total])
    assert (Qr[total:] == 9).all()
    want = turned(K, positions, freqs, 0, 1.0)
    written = torch.zeros(sum(slots), dtype=torch.bool)
    t, c = starts(new), starts(slots)
    for s, (n, h, r) in enumerate(zip(new, have, room)):
        for j in range(min(n, r)):
            at = c[s] + h + j
            written[at] = True
            close(Kc[:, at], want[t[s] + j])
            assert torch.equal(Vc[:, at], V[t[s] + j]) and (pos[:, at] == positions[t[s] + j]).all()
    for x in (Kc, Vc, norms, pos):
        assert (x[:, ~written.to(DEV)] == 9).all()
    again = torch.empty_like(norms)
    l2kv.l2kv_norms(Kc, again)
    assert torch.equal(norms[:, written.to(DEV)], again[:, written.to(DEV)])


def test_like_append_without_a_turn():
    """At position 0 it is l2kv_stream_append."""
    Hkv, D, n = 4, 128, 3
    _, K, V = inputs(1, n, 1, Hkv, D, torch.bfloat16)
    zero = torch.zeros(n, dtype=torch.int32, device=DEV)
    lens = torch.tensor([1, 0, 2], dtype=torch.int32, device=DEV)
    a, b = cache(Hkv, 9, D, torch.bfloat16), cache(Hkv, 9, D, torch.bfloat16)
    out_a, out_b = torch.empty_like(lens), torch.empty_like(lens)
    l2kv.l2kv_rotary_append(None, K, V, zero, l2kv.l2kv_rotary_freqs(64).to(DEV), None, *a, offsets([1, 1, 1]), offsets([3, 3, 3]), lens, out_a)
    l2kv.l2kv_stream_append(K.contiguous().unsqueeze(0), V.contiguous().unsqueeze(0), zero, offsets([3, 3, 3]), lens, out_b, *b)
    for x, y in zip(a + (out_a,), b + (out_b,)):
        assert torch.equal(x, y)


def test_angles_of_far_positions():
    """A whole turn too much or too little would show: fp32 angles are off by a tenth of a radian here."""
    D = 64
    positions = torch.tensor([2 ** 20 + 1, 2 ** 24 + 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).to(torch.int32).to(DEV)
    freqs = l2kv.l2kv_rotary_freqs(D).to(DEV)
    K = torch.ones((4, 1, D), device=DEV)
    Kc, Vc, norms, pos = cache(1, 4, D, torch.float32)
    l2kv.l2kv_rotary_append(None, K, K, positions, freqs, None, Kc, Vc, norms, pos)
    # the product of position and frequency is rounded to 2^-53 of itself on both sides
    close(Kc.transpose(0, 1), turned(K, positions, freqs, 0, 1.0), far=2 ** 31 * 2.0 ** -52)


def test_inconsistent_arrays_stay_inside():
    Hkv, D = 2, 128
    Q, K, V = inputs(2, 20, 2, Hkv, D, torch.bfloat16)
    positions, freqs = torch.arange(20, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(D).to(DEV)
    for tokens in ([0, 30, 10], [-4, 5, 1 << 40], [9, 3, 0]):
        for slots in ([0, 50, 20], [-9, 3, 1 << 40], [12, 8, 0]):
            for lens in ([0, 0], [-5, 1 << 30]):
                Qr = torch.full((22, 2, D), 3.0, dtype=torch.bfloat16, device=DEV)
                Kc, Vc = (torch.full((Hkv * 12 + 2, D), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
                _, _, norms, pos = cache(Hkv, 12, D, torch.bfloat16)
                l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr[1:21], Kc[1:-1].view(Hkv, 12, D), Vc[1:-1].view(Hkv, 12, D), norms, pos,
                                        *(torch.tensor(x, device=DEV) for x in (tokens, slots)), torch.tensor(lens, dtype=torch.int32, device=DEV))
                assert all((x[0] == 3).all() and (x[-1] == 3).all() for x in (Qr, Kc, Vc))


def test_many_tokens_and_a_graph():
    total, Hq, Hkv, D = 3001, 4, 2, 64
    Q, K, V = inputs(3, total, Hq, Hkv, D, torch.float32)
    Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    positions, freqs = torch.arange(total, dtype=torch.int32, device=DEV), l2kv.l2kv_rotary_freqs(32).to(DEV)
    Qr, c = torch.empty_like(Q), cache(Hkv, total, D, torch.float32)

    def call():
        l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, *c, layout=1)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        for t in (Q, K, V):
            t.copy_(randn(torch.Generator(device=DEV).manual_seed(seed), *t.shape))
        Qr.zero_(), c[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        close(Qr, turned(Q, positions, freqs, 1, 1.0))
        close(c[0].transpose(0, 1), turned(K, positions, freqs, 1, 1.0))


@pytest.mark.parametrize("dtype,D", ROWS)
@pytest.mark.parametrize("Hq,Hkv,total", [(1, 1, 4099), (4, 1, 4111), (2, 2, 4096), (6, 3, 2051), (1, 1, 1029)])
@pytest.mark.parametrize("layout", [0, 1])
def test_many_tokens_of_few_heads(dtype, D, Hq, Hkv, total, layout):
    """Workgroups of 16, 8 and 4 tokens, the last one not full; into rows as they are, and into the slots of many sequences."""
    Q, K, V = inputs(total, total, Hq, Hkv, D, dtype)
    positions = (torch.arange(total, dtype=torch.int32) % 1000 * 77).to(DEV)
    rot = 32
    freqs = l2kv.l2kv_rotary_freqs(rot, 10000.0).to(DEV)
    Qr = torch.empty((total, Hq, D), dtype=dtype, device=DEV)
    Kc, Vc, norms, pos = cache(Hkv, total, D, dtype)
    l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, Kc, Vc, norms, pos, layout=layout)
    close(Qr, turned(Q, positions, freqs, layout, 1.0))
    close(Kc.transpose(0, 1), turned(K, positions, freqs, layout, 1.0))
    assert torch.equal(Vc, V.transpose(0, 1)) and torch.equal(pos, positions.expand(Hkv, total))
    again = torch.empty_like(norms)
    l2kv.l2kv_norms(Kc, again)
    assert torch.equal(norms, again)
    new = [7] * (total // 7) + [total % 7]
    slots = [n + 3 for n in new]
    Ks, Vs, norms_s, pos_s = cache(Hkv, sum(slots), D, dtype)
    lens_in = torch.full((len(new),), 2, dtype=torch.int32, device=DEV)
    lens_out = torch.empty_like(lens_in)
    l2kv.l2kv_rotary_append(Q, K, V, positions, freqs, Qr, Ks, Vs, norms_s, pos_s, offsets(new), offsets(slots), lens_in, lens_out, layout=layout)
    assert lens_out.tolist() == [n + 2 for n in new]
    to = torch.cat([torch.arange(n) + 2 + c for n, c in zip(new, starts(slots))]).to(DEV)
    assert torch.equal(Ks[:, to], Kc) and torch.equal(Vs[:, to], Vc) and torch.equal(norms_s[:, to], norms) and torch.equal(pos_s[:, to], pos)
    free = torch.ones(sum(slots), dtype=torch.bool, device=DEV)
    free[to] = False
    assert (Ks[:, free] == 9).all() and (Vs[:, free] == 9).all() and (norms_s[:, free] == 9).all() and (pos_s[:, free] == 9).all()
