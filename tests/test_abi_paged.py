"""Refusals of the calls of the cache in pages: no device is touched."""
import math

import pytest
import torch

import paper_2406_11430_amd as l2kv
from test_abi_rows import E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_WS, ODD, P, ROTARY, call

APPEND = {k: v for k, v in ROTARY.items() if k not in ("token_off", "slot_off", "lens_in", "lens_out", "slots", "positions", "freqs", "rot", "layout",
                                                      "amplitude", "n_seq", "Qr", "Kc", "Vc", "norms", "pos", "stream")}
NORM = {**APPEND, "qw": P, "kw": P, "eps": 1e-6, **{k: ROTARY[k] for k in ("positions", "freqs", "rot", "layout", "amplitude", "n_seq", "token_off", "slot_off", "lens_in",
                                                                          "lens_out", "slots", "Qr", "Kc", "Vc", "norms", "pos", "stream")}}
BOTH = [(E_NULL, dict(K=None)), (E_NULL, dict(V=None)), (E_NULL, dict(Q=None)), (E_NULL, dict(Qr=None)), (E_NULL, dict(positions=None)),
        (E_NULL, dict(freqs=None)), (E_NULL, dict(Kc=None)), (E_NULL, dict(Vc=None)), (E_NULL, dict(norms=None)), (E_NULL, dict(pos=None)),
        (E_DTYPE, dict(dt=2)), (E_SHAPE, dict(total=0)), (E_SHAPE, dict(Hq=0)), (E_SHAPE, dict(Hkv=0)), (E_SHAPE, dict(D=96)), (E_SHAPE, dict(D=256, dt=0)),
        (E_SHAPE, dict(rot=24)), (E_SHAPE, dict(rot=144)), (E_SHAPE, dict(layout=2)), (E_SHAPE, dict(amplitude=math.nan)), (E_SHAPE, dict(eps=-1e-9)),
        (E_SHAPE, dict(eps=math.inf)), (E_SHAPE, dict(eps=math.nan)), (E_SHAPE, dict(k_stride=0)), (E_ALIGN, dict(qw=P + 2)), (E_ALIGN, dict(kw=P + 1)),
        (E_ALIGN, dict(Kc=ODD)), (E_ALIGN, dict(q_stride=516))]


@pytest.mark.parametrize("want,kw", BOTH + [(E_SHAPE, dict(slots=7)), (E_NULL, dict(token_off=P, n_seq=1)),
                                            (E_SHAPE, dict(token_off=P, slot_off=P, lens_in=P, lens_out=P, n_seq=1))])
def test_norm_rotary_append_refuses(want, kw):
    assert call("l2kv_norm_rotary_append", NORM, **kw) == want


PAGED = {**APPEND, "qw": P, "kw": P, "eps": 1e-6, "positions": P, "freqs": P, "rot": 64, "layout": 0, "amplitude": 1.0, "n_seq": 2, "token_off": P, "table": P,
         "max_pages": 4, "page": 16, "n_pages": 8, "lens_in": P, "lens_out": P + 64, "Qr": P, "Kc": P, "Vc": P, "norms": P, "pos": P, "stream": None}
PAGES_BAD = [(E_SHAPE, dict(page=p)) for p in (0, -16, 8, 24, 48, 512)] + [
    (E_SHAPE, dict(max_pages=0)), (E_SHAPE, dict(n_pages=0)), (E_SHAPE, dict(n_pages=1 << 28)), (E_SHAPE, dict(max_pages=1 << 28)), (E_SHAPE, dict(n_seq=0))]


@pytest.mark.parametrize("want,kw", BOTH + PAGES_BAD + [(E_NULL, dict(token_off=None)), (E_NULL, dict(table=None)), (E_NULL, dict(lens_in=None)),
                                                        (E_SHAPE, dict(lens_out=P)), (E_ALIGN, dict(table=P + 2)), (E_ALIGN, dict(token_off=ODD)),
                                                        (E_SHAPE, dict(n_seq=1 << 30))])
def test_paged_append_refuses(want, kw):
    assert call("l2kv_paged_append", PAGED, **kw) == want


ATTN = dict(Q=P, K=P, V=P, dt=1, n_seq=1, Hq=4, Hkv=2, D=128, total=100, q_stride=512, q_off=P, table=P, max_pages=10, page=16, n_pages=20, kv_lens=P,
            max_kv=100, scale=0.0, O=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("want,kw", PAGES_BAD + [(E_NULL, {k: None}) for k in ("Q", "K", "V", "O", "q_off", "table", "kv_lens")] + [
    (E_DTYPE, dict(dt=-1)), (E_SHAPE, dict(Hq=5)), (E_SHAPE, dict(Hq=18)), (E_SHAPE, dict(Hkv=0)), (E_SHAPE, dict(D=32)), (E_SHAPE, dict(total=0)),
    (E_SHAPE, dict(q_stride=256)), (E_SHAPE, dict(max_kv=161)), (E_SHAPE, dict(max_kv=0)), (E_SHAPE, dict(scale=math.inf)), (E_SHAPE, dict(D=256, Hq=10, q_stride=2560)),
    (E_ALIGN, dict(q_stride=516)), (E_ALIGN, dict(Q=ODD)), (E_ALIGN, dict(K=ODD)), (E_ALIGN, dict(V=ODD)), (E_ALIGN, dict(O=ODD)), (E_ALIGN, dict(ws=ODD)),
    (E_ALIGN, dict(q_off=ODD)), (E_ALIGN, dict(table=P + 2)), (E_ALIGN, dict(kv_lens=P + 2)), (E_WS, dict(ws_bytes=1000)), (E_WS, dict(ws=None))])
def test_paged_attn_refuses(want, kw):
    defaults = {**ATTN, "total": 1, "max_kv": 9000, "max_pages": 600, "n_pages": 600} if want == E_WS else ATTN        # one row over many keys
    assert call("l2kv_paged_attn", defaults, **kw) == want


INIT = dict(table=P, n_seq=2, max_pages=4, refs=P, free=P, count=P, n_pages=8, stream=None)
FORK = dict(table=P, lens=P, n_seq=2, parents=P, n_out=3, max_pages=4, page=16, n_pages=8, out=P + 64, lens_out=P + 128, refs=P, stream=None)
RESERVE = dict(table=P, n_seq=2, max_pages=4, page=16, first=P, to=P, ends=P + 64, refs=P, free=P, count=P, n_pages=8, dt=1, planes=2, D=128, K=P, V=P, norms=P,
               pos=P, ws=P, ws_bytes=144, stream=None)
RELEASE = dict(table=P, n_seq=2, max_pages=4, page=16, keep=P, refs=P, free=P, count=P, n_pages=8, ws=P, ws_bytes=144, stream=None)
COMPRESS = dict(K=P, V=P, norms=P, pos=P, dt=1, planes=2, n_seq=2, D=128, page=16, n_pages=8, table=P, max_pages=4, lens=P, keep=P, out=P + 64, max_out=4,
                lens_out=P + 128, rows=100, kept=50, max_len=60, ws=P, ws_bytes=1 << 20, stream=None)
POINTERS = {"l2kv_pages_init": (INIT, ("table", "refs", "free", "count")), "l2kv_pages_fork": (FORK, ("table", "lens", "parents", "out", "lens_out", "refs")),
            "l2kv_pages_reserve": (RESERVE, ("table", "first", "to", "ends", "refs", "free", "count", "K", "V", "norms", "pos")),
            "l2kv_pages_release": (RELEASE, ("table", "keep", "refs", "free", "count")),
            "l2kv_paged_compress": (COMPRESS, ("K", "V", "norms", "pos", "table", "lens", "keep", "out", "lens_out"))}


@pytest.mark.parametrize("name", POINTERS)
def test_pages_refuse(name):
    defaults, pointers = POINTERS[name]
    for p in pointers:
        assert call(name, defaults, **{p: None}) == E_NULL, p
        assert call(name, defaults, **{p: defaults[p] + 2}) == E_ALIGN, p
    books = [(E_SHAPE, dict(n_seq=65536))] + ([(E_SHAPE, dict(n_seq=1 << 10, max_pages=(1 << 20) + 1))] if name != "l2kv_paged_compress" else [])
    for want, kw in PAGES_BAD + books:
        if set(kw) <= set(defaults):
            assert call(name, defaults, **kw) == want, kw
    if "ws" in defaults:
        for kw in (dict(ws=None), dict(ws_bytes=140)):
            assert call(name, defaults, **kw) == E_WS
        assert call(name, defaults, ws=ODD) == E_ALIGN
    if "dt" in defaults:
        assert call(name, defaults, dt=3) == E_DTYPE and call(name, defaults, D=80) == E_SHAPE and call(name, defaults, planes=0) == E_SHAPE


@pytest.mark.parametrize("name,kw", [("l2kv_pages_fork", dict(out=P)), ("l2kv_pages_fork", dict(lens_out=P)), ("l2kv_pages_fork", dict(n_out=0)),
                                     ("l2kv_pages_fork", dict(n_out=65536)), ("l2kv_pages_fork", dict(n_out=1 << 10, max_pages=(1 << 20) + 1)),
                                     ("l2kv_pages_reserve", dict(ends=P)), ("l2kv_paged_compress", dict(out=P)),
                                     ("l2kv_paged_compress", dict(lens_out=P)), ("l2kv_paged_compress", dict(rows=0)), ("l2kv_paged_compress", dict(kept=0)),
                                     ("l2kv_paged_compress", dict(kept=1 << 29)), ("l2kv_paged_compress", dict(max_len=101)), ("l2kv_paged_compress", dict(max_len=0)),
                                     ("l2kv_paged_compress", dict(max_out=0)), ("l2kv_paged_compress", dict(planes=1 << 30))])
def test_sizes_and_aliases_refused(name, kw):
    assert call(name, POINTERS[name][0], **kw) == E_SHAPE


def test_workspaces_of_bad_sizes():
    assert l2kv.l2kv_pages_workspace_bytes(8) == 144 and l2kv.l2kv_pages_workspace_bytes(0) == l2kv.l2kv_pages_workspace_bytes(1 << 31) == 0
    f = l2kv.l2kv_paged_compress_workspace_bytes
    assert f(2, 3, 100, 50) > 0 and f(0, 3, 100, 50) == f(2, 0, 100, 50) == f(2, 3, 0, 50) == f(2, 3, 100, 0) == f(2, 3, 1 << 31, 50) == f(2, 3, 100, 1 << 29) == 0
    g = l2kv.l2kv_paged_attn_workspace_bytes
    assert g(1, 5, 2, 10, 10, 128, 1) == g(0, 4, 2, 10, 10, 128, 1) == 0 and g(1, 32, 8, 1, 100000, 128, torch.bfloat16) > 0


def test_host_tensors_are_refused():
    Q, K = torch.zeros((3, 4, 64)), torch.zeros((2, 32, 64))
    off, n, t, w = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(64)
    norms, pos, refs = K[..., 0], K[..., 0].int(), torch.zeros(2, dtype=torch.int32)
    freqs = torch.zeros(16, dtype=torch.float64)
    for f in (lambda: l2kv.l2kv_paged_attn(Q, K, K, off, t, 16, n, 3, Q, None),
              lambda: l2kv.l2kv_paged_append(Q, Q[:, :2], Q[:, :2], pos[0, :3], freqs, Q, K, K, norms, pos, off, t, 16, n, None, w, w),
              lambda: l2kv.l2kv_norm_rotary_append(Q, Q[:, :2], Q[:, :2], w, w, 0.0, pos[0, :3], freqs, Q, K, K, norms, pos),
              lambda: l2kv.l2kv_pages_init(t, refs, refs, n), lambda: l2kv.l2kv_pages_fork(t, n, n, t, n, refs, 16),
              lambda: l2kv.l2kv_pages_reserve(t, n, n, n, refs, refs, n, 16, K, K, norms, pos, K),
              lambda: l2kv.l2kv_pages_release(t, n, refs, refs, n, 16, K),
              lambda: l2kv.l2kv_paged_compress(K, K, norms, pos, t, n, n, t, n, 16, 5, 3, 5, K)):
        with pytest.raises(ValueError, match="device tensors"):
            f()
