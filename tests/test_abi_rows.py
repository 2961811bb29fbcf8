"""Refusals of the calls around the compressed cache, and the host's frequencies: no device is touched."""
import ctypes as C
import math

import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding

OK, E_NULL, E_SHAPE, E_DTYPE, E_WS, E_ALIGN = 0, -1, -2, -3, -5, -6
P, ODD = 0x1000, 0x1004                    # fake device addresses, never dereferenced: 16-byte aligned, and not


def call(name, defaults, **kw):
    assert not set(kw) - set(defaults)
    return getattr(binding.lib(), name)(*{**defaults, **kw}.values())


ROTARY = dict(Q=P, K=P, V=P, dt=1, total=8, Hq=4, Hkv=2, D=128, q_stride=512, k_stride=256, v_stride=256, positions=P, freqs=P, rot=64, layout=0,
              amplitude=1.0, n_seq=0, token_off=None, slot_off=None, lens_in=None, lens_out=None, slots=8, Qr=P, Kc=P, Vc=P, norms=P, pos=P,
              stream=None)


@pytest.mark.parametrize("want,kw", [
    (E_NULL, dict(K=None)), (E_NULL, dict(V=None)), (E_NULL, dict(Q=None)), (E_NULL, dict(Qr=None)), (E_NULL, dict(positions=None)),
    (E_NULL, dict(freqs=None)), (E_NULL, dict(Kc=None)), (E_NULL, dict(Vc=None)), (E_NULL, dict(norms=None)), (E_NULL, dict(pos=None)),
    (E_NULL, dict(token_off=P, n_seq=1)), (E_NULL, dict(token_off=P, slot_off=P, n_seq=1)), (E_NULL, dict(lens_in=P)), (E_NULL, dict(lens_out=P)),
    (E_DTYPE, dict(dt=2)), (E_SHAPE, dict(total=0)), (E_SHAPE, dict(total=1 << 31)), (E_SHAPE, dict(Hq=0)), (E_SHAPE, dict(Hkv=0)), (E_SHAPE, dict(Hq=70000)),
    (E_SHAPE, dict(D=96)), (E_SHAPE, dict(D=256, dt=0)), (E_SHAPE, dict(rot=0)), (E_SHAPE, dict(rot=24)), (E_SHAPE, dict(rot=144)), (E_SHAPE, dict(layout=2)),
    (E_SHAPE, dict(amplitude=math.inf)), (E_SHAPE, dict(slots=7)), (E_SHAPE, dict(slots=0)), (E_SHAPE, dict(q_stride=504)), (E_SHAPE, dict(k_stride=0)),
    (E_SHAPE, dict(v_stride=1 << 60)), (E_SHAPE, dict(token_off=P, slot_off=P, lens_in=P, n_seq=0)),
    (E_SHAPE, dict(token_off=P, slot_off=P, lens_in=P, lens_out=P, n_seq=1)),
    (E_ALIGN, dict(q_stride=516)), (E_ALIGN, dict(k_stride=258)), (E_ALIGN, dict(Q=ODD)), (E_ALIGN, dict(K=ODD)), (E_ALIGN, dict(Qr=ODD)), (E_ALIGN, dict(Kc=ODD)),
    (E_ALIGN, dict(freqs=ODD)), (E_ALIGN, dict(norms=P + 2)), (E_ALIGN, dict(token_off=ODD, slot_off=P, lens_in=P, n_seq=1)),
])
def test_rotary_append_refuses(want, kw):
    assert call("l2kv_rotary_append", ROTARY, **kw) == want


PROMPT = dict(Q=P, K=P, V=P, dt=1, n_seq=1, Hq=4, Hkv=2, D=128, total=100, q_stride=512, q_off=P, rows=100, head_stride=12800, kv_off=P, kv_lens=None,
              max_kv=100, scale=0.0, O=P, ws=P, ws_bytes=1 << 30, stream=None)
ROWS_BAD = [
    (E_NULL, dict(Q=None)), (E_NULL, dict(K=None)), (E_NULL, dict(V=None)), (E_NULL, dict(O=None)), (E_NULL, dict(q_off=None)), (E_NULL, dict(kv_off=None)),
    (E_DTYPE, dict(dt=-1)), (E_SHAPE, dict(n_seq=0)), (E_SHAPE, dict(Hq=5)), (E_SHAPE, dict(Hq=18)), (E_SHAPE, dict(Hkv=0)), (E_SHAPE, dict(D=32)),
    (E_SHAPE, dict(total=0)), (E_SHAPE, dict(total=1 << 31)), (E_SHAPE, dict(q_stride=256)), (E_SHAPE, dict(rows=0)), (E_SHAPE, dict(rows=1 << 31)),
    (E_SHAPE, dict(max_kv=101)), (E_SHAPE, dict(max_kv=-1)), (E_SHAPE, dict(head_stride=0)), (E_SHAPE, dict(head_stride=1 << 60)), (E_SHAPE, dict(scale=math.nan)),
    (E_SHAPE, dict(n_seq=1 << 24)), (E_SHAPE, dict(D=256, Hq=10, q_stride=2560)),
    (E_ALIGN, dict(q_stride=516)), (E_ALIGN, dict(head_stride=12804)), (E_ALIGN, dict(Q=ODD)), (E_ALIGN, dict(K=ODD)), (E_ALIGN, dict(V=ODD)), (E_ALIGN, dict(O=ODD)),
    (E_ALIGN, dict(ws=ODD)), (E_ALIGN, dict(q_off=ODD)), (E_ALIGN, dict(kv_off=ODD)), (E_ALIGN, dict(kv_lens=P + 2)), (E_WS, dict(ws_bytes=1000)), (E_WS, dict(ws=None)),
]


@pytest.mark.parametrize("want,kw", ROWS_BAD + [(E_SHAPE, dict(max_kv=0))])
def test_prompt_attn_refuses(want, kw):
    defaults = {**PROMPT, "total": 4, "rows": 9000, "max_kv": 9000} if want == E_WS else PROMPT          # few rows over many keys
    assert call("l2kv_prompt_attn", defaults, **kw) == want


TREE = dict(Q=P, K=P, V=P, Kt=P, Vt=P, dt=1, n_seq=1, Hq=4, Hkv=2, D=128, total=100, q_stride=512, q_off=P, mask=P, words=4, rows=100, head_stride=12800,
            kv_off=P, kv_lens=P, max_kv=100, scale=0.0, O=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("want,kw", ROWS_BAD + [(E_NULL, dict(Kt=None)), (E_NULL, dict(Vt=None)), (E_NULL, dict(mask=None)), (E_NULL, dict(kv_lens=None)),
                                                (E_SHAPE, dict(words=0)), (E_ALIGN, dict(Kt=ODD)), (E_ALIGN, dict(mask=P + 2))])
def test_tree_attn_refuses(want, kw):
    defaults = {**TREE, "total": 4, "rows": 9000, "max_kv": 9000} if want == E_WS else TREE
    assert call("l2kv_tree_attn", defaults, **kw) == want


PATH = dict(Kt=P, Vt=P, norms_t=P, pos_t=P, dt=1, planes=2, n_seq=1, D=128, total=8, node_off=P, path=P, max_path=4, path_lens=P, slot_off=P, slots=20,
            lens_in=P, lens_out=P + 64, Kc=P, Vc=P, norms_c=P, pos_c=P, stream=None)


@pytest.mark.parametrize("want,kw", [(E_NULL, {k: None}) for k in ("Kt", "Vt", "norms_t", "pos_t", "node_off", "path", "path_lens", "slot_off", "lens_in",
                                                                   "lens_out", "Kc", "Vc", "norms_c", "pos_c")] + [
    (E_DTYPE, dict(dt=9)), (E_SHAPE, dict(planes=0)), (E_SHAPE, dict(n_seq=0)), (E_SHAPE, dict(n_seq=1 << 24)), (E_SHAPE, dict(D=80)), (E_SHAPE, dict(total=0)),
    (E_SHAPE, dict(max_path=0)), (E_SHAPE, dict(slots=0)), (E_SHAPE, dict(lens_out=P)), (E_ALIGN, dict(Kt=ODD)), (E_ALIGN, dict(Vc=ODD)), (E_ALIGN, dict(node_off=ODD)),
    (E_ALIGN, dict(path=P + 2))])
def test_append_path_refuses(want, kw):
    assert call("l2kv_stream_append_path", PATH, **kw) == want


def test_workspaces_of_bad_sizes():
    for f in (l2kv.l2kv_prompt_attn_workspace_bytes, l2kv.l2kv_tree_attn_workspace_bytes):
        assert f(0, 4, 2, 10, 10, 128, 1) == f(1, 5, 2, 10, 10, 128, 1) == f(1, 4, 2, 0, 10, 128, 1) == f(1, 4, 2, 10, 10, 100, 1) == f(1, 4, 2, 10, 10, 128, 7) == 0
        assert f(1, 32, 8, 1, 100000, 128, torch.bfloat16) > 0
        assert f(100000, 32, 8, 1, 100000, 128, torch.bfloat16) < 1 << 31             # empty sequences take no room for keys in shares


@pytest.mark.parametrize("R", [16, 64, 128, 256])
def test_frequencies(R):
    i = torch.arange(R // 2, dtype=torch.float64)
    f = 10000.0 ** (-2 * i / R)
    plain = l2kv.l2kv_rotary_freqs(R)
    assert torch.allclose(plain, f, rtol=1e-14, atol=0)
    assert torch.allclose(l2kv.l2kv_rotary_freqs(R, 10000.0, binding.L2KV_ROTARY_LINEAR, 4.0), f / 4, rtol=1e-14, atol=0)
    base = l2kv.l2kv_rotary_freqs(R, 10000.0, binding.L2KV_ROTARY_BASE, 4.0)
    assert base[0] == 1 and torch.allclose(base[-1], f[-1] / 4, rtol=1e-13, atol=0) and (base.diff() < 0).all()
    bands = l2kv.l2kv_rotary_freqs(R, 10000.0, binding.L2KV_ROTARY_BANDS, 4.0, 4096, 1.0, 32.0)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(bands[turns >= 32], plain[turns >= 32]) and torch.allclose(bands[turns <= 1], f[turns <= 1] / 4, rtol=1e-14, atol=0)
    ramp = (turns > 1) & (turns < 32)
    keep = (turns[ramp] - 1) / 31
    assert torch.allclose(bands[ramp], f[ramp] * keep + f[ramp] / 4 * (1 - keep), rtol=1e-13, atol=0)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=272), dict(rot_dim=64, base=0.0), dict(rot_dim=64, base=math.inf),
                                dict(rot_dim=64, scaling=4), dict(rot_dim=64, scaling=1, factor=0.0), dict(rot_dim=64, scaling=2, factor=math.nan),
                                dict(rot_dim=64, scaling=3, factor=2.0), dict(rot_dim=64, scaling=3, factor=2.0, original_len=100, low=4.0, high=4.0),
                                dict(rot_dim=64, scaling=3, factor=2.0, original_len=100, low=-1.0)])
def test_frequencies_refused(kw):
    with pytest.raises(l2kv.L2KVError):
        l2kv.l2kv_rotary_freqs(**kw)
    assert binding.lib().l2kv_rotary_freqs(64, 1e4, 0, 1.0, 0, 1.0, 32.0, None) == E_NULL


def test_host_tensors_are_refused():
    Q = torch.zeros((3, 4, 64))
    K = torch.zeros((2, 3, 64))
    off, ints = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        l2kv.l2kv_prompt_attn(Q, K, K, off, off, None, 3, Q, None)
    with pytest.raises(ValueError, match="device tensors"):
        l2kv.l2kv_tree_attn(Q, K, K, ints, off, 3, K, K, off, ints, Q, None)
    with pytest.raises(ValueError, match="device tensors"):
        l2kv.l2kv_rotary_append(Q, Q[:, :2], Q[:, :2], ints, off.double(), Q, K, K, K[..., 0], K[..., 0].int())
