"""The native calls of the cache in pages: the same results as through ctypes, and what they do not take is left to the checks in Python."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding
from test_binding_calls_rows import DEV, Taken, ints, longs, rand, rotary

NAMES = {"norm_rotary_append": 21, "paged_append": 22, "paged_attn": 13, "pages_fork": 9, "pages_reserve": 15, "pages_release": 9, "paged_compress": 16}


def test_what_is_not_a_device_tensor_is_left_to_the_checks():
    native = binding.calls()
    for name, n in NAMES.items():
        call = getattr(native, name)
        assert call() is None and call(*range(n)) is None
        assert call(*[None] * (n - 1), binding._stream) is None
        assert call(*[torch.zeros((2, 2, 64))] * (n - 1), binding._stream) is None


def weight():
    return torch.linspace(0.5, 1.5, 64, device=DEV)


def cache():
    return dict(Kc=rand(5, 2, 64, 64), Vc=rand(6, 2, 64, 64), norms_c=rand(7, 2, 64).float(), pos_c=torch.arange(128, dtype=torch.int32, device=DEV).view(2, 64))


def norm(**kw):
    a, outs = rotary(q_weight=weight(), k_weight=weight() * 2, eps=1e-3)
    a.update(kw)
    return a, outs


def append(**kw):
    qkv = rand(0, 5, 8, 64)
    a = dict(Q=qkv[:, :4], K=qkv[:, 4:6], V=qkv[:, 6:], positions=ints(1, 2, 3, 4, 5), freqs=l2kv.l2kv_rotary_freqs(32, 10000.0).to(DEV),
             Qr=torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=DEV), **cache(), token_offsets=longs(0, 2, 5), page_table=ints(0, 2, 3, -1).view(2, 2),
             page_size=16, lens_in=ints(15, 4), lens_out=ints(0, 0), q_weight=weight(), k_weight=weight(), eps=1e-5, layout=1, amplitude=1.5)
    a.update(kw)
    return a, ("Qr", "Kc", "Vc", "norms_c", "pos_c", "lens_out")


def attn(**kw):
    c = cache()
    a = dict(Q=rand(0, 5, 8, 64)[:, :4], Kc=c["Kc"], Vc=c["Vc"], q_offsets=longs(0, 4, 5), page_table=ints(1, 2, 3, -1).view(2, 2), page_size=16,
             kv_lens=ints(30, 12), max_kv=30, O=torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=DEV), workspace=None, scale=0.3)
    a.update(kw)
    return a, ("O",)


def pool():
    return dict(refs=ints(1, 1, 1, 0), free_pages=ints(3, 0, 0, 0), free_count=ints(1), page_size=16)


def fork(**kw):
    a = dict(table_in=ints(0, 1, 2, -1).view(2, 2), lens_in=ints(20, 3), parents=ints(1, 0, 0), table_out=ints(*[7] * 6).view(3, 2), lens_out=ints(0, 0, 0),
             refs=ints(1, 1, 1, 0), page_size=16)
    a.update(kw)
    return a, ("table_out", "lens_out", "refs")


def workspace(n):
    return torch.zeros(n, dtype=torch.uint8, device=DEV)


def reserve(**kw):
    a = dict(page_table=ints(0, 1, 2, -1).view(2, 2), first=ints(20, 3), to=ints(21, 17), ends=ints(0, 0), **pool(), **cache(), workspace=workspace(80))
    a.update(kw)
    return a, ("page_table", "ends", "refs", "free_pages", "free_count", "Kc", "pos_c")


def release(**kw):
    a = dict(page_table=ints(0, 1, 2, -1).view(2, 2), keep_lens=ints(16, 0), **pool(), workspace=workspace(80))
    a.update(kw)
    return a, ("page_table", "refs", "free_pages", "free_count")


def compress(**kw):
    a = dict(**cache(), table_in=ints(0, 1, 2, -1).view(2, 2), lens_in=ints(20, 9), keep=ints(9, 5), table_out=ints(3, -1, -1, -1).view(2, 2), lens_out=ints(0, 0),
             page_size=16, total_rows=30, total_kept=14, max_len=20, workspace=workspace(1024))
    a.update(kw)
    return a, ("Kc", "Vc", "norms_c", "pos_c", "lens_out")


CALLS = {"norm_rotary_append": (norm, l2kv.l2kv_norm_rotary_append), "paged_append": (append, l2kv.l2kv_paged_append), "paged_attn": (attn, l2kv.l2kv_paged_attn),
         "pages_fork": (fork, l2kv.l2kv_pages_fork), "pages_reserve": (reserve, l2kv.l2kv_pages_reserve), "pages_release": (release, l2kv.l2kv_pages_release),
         "paged_compress": (compress, l2kv.l2kv_paged_compress)}


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("without", [False, True])
def test_both_ways_are_the_same(name, without, monkeypatch):
    build, entry = CALLS[name]
    kw = {}
    if without:
        kw = {"norm_rotary_append": dict(Q=None, Qr=None, q_weight=None), "paged_append": dict(Q=None, Qr=None, q_weight=None, k_weight=None, lens_out=None, eps=0),
              "paged_attn": dict(workspace=workspace(1 << 20), scale=0)}.get(name, {})
    native, outputs = Taken(binding.calls()), []
    for calls in (native, binding._PythonCalls):
        monkeypatch.setattr(binding, "_calls", calls)
        a, outs = build(**{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
        entry(**a, stream=torch.cuda.current_stream())
        outputs.append([a[o].clone() for o in outs if a[o] is not None])
    assert native.count == 1
    for x, y in zip(*outputs):
        assert torch.equal(x, y) and (x.numel() == 1 or x.abs().sum() > 0)          # (the last free page may be gone)


WRONG = [(name, key, change) for name in NAMES for key, change in {
    "norm_rotary_append": [("Q", "half"), ("q_weight", "half"), ("q_weight", "short"), ("k_weight", "cpu"), ("K", "heads"), ("Kc", "short"), ("lens_in", "long")],
    "paged_append": [("Q", "half"), ("K", "heads"), ("K", "float"), ("V", "float"), ("positions", "long"), ("freqs", "float"), ("Qr", "short"), ("Kc", "turned"), ("Vc", "half"),
                     ("norms_c", "short"), ("pos_c", "long"), ("token_offsets", "int"), ("token_offsets", "short"), ("page_table", "long"), ("page_table", "short"),
                     ("page_table", "cpu"), ("lens_in", "short"), ("lens_out", "long"), ("q_weight", "half"), ("k_weight", "short")],
    "paged_attn": [("Q", "half"), ("Q", "heads"), ("Kc", "float"), ("Vc", "short"), ("q_offsets", "int"), ("q_offsets", "short"), ("page_table", "long"), ("page_table", "turned"),
                   ("kv_lens", "long"), ("kv_lens", "short"), ("O", "float"), ("O", "short"), ("Kc", "cpu")],
    "pages_fork": [("table_in", "long"), ("lens_in", "short"), ("parents", "long"), ("parents", "short"), ("table_out", "short"), ("lens_out", "short"), ("refs", "long"),
                   ("refs", "cpu")],
    "pages_reserve": [("page_table", "long"), ("first", "short"), ("to", "long"), ("ends", "short"), ("refs", "short"), ("free_pages", "short"), ("free_count", "long"),
                      ("Kc", "short"), ("Vc", "float"), ("norms_c", "short"), ("pos_c", "long"), ("workspace", "cpu")],
    "pages_release": [("page_table", "long"), ("keep_lens", "short"), ("refs", "long"), ("free_pages", "short"), ("free_count", "long"), ("workspace", "cpu")],
    "paged_compress": [("Kc", "half"), ("Vc", "short"), ("norms_c", "short"), ("pos_c", "long"), ("table_in", "long"), ("lens_in", "short"), ("keep", "long"),
                       ("table_out", "short"), ("lens_out", "short"), ("workspace", "cpu")]}[name]]


@pytest.mark.gpu
@pytest.mark.parametrize("name,key,change", WRONG)
def test_wrong_arguments_are_refused(name, key, change):
    build, entry = CALLS[name]
    a, _ = build()
    x = a[key]
    a[key] = {"half": lambda: x.half(), "float": lambda: x.float(), "long": lambda: x.long(), "int": lambda: x.int(), "cpu": lambda: x.cpu(),
              "short": lambda: x[:-1].contiguous(), "turned": lambda: x.transpose(-1, -2).contiguous().transpose(-1, -2),
              "heads": lambda: torch.cat([x, x], -1)[..., :x.shape[-1]]}[change]()
    with pytest.raises((AssertionError, TypeError, ValueError)):
        entry(**a)


@pytest.mark.gpu
def test_pages_that_do_not_divide_the_slots():
    for build, entry in ((append, l2kv.l2kv_paged_append), (attn, l2kv.l2kv_paged_attn), (compress, l2kv.l2kv_paged_compress)):
        for size in (0, -16, 48):
            with pytest.raises(ValueError, match="whole pages"):
                entry(**build(page_size=size)[0])
        with pytest.raises(l2kv.L2KVError):
            entry(**build(page_size=8)[0])
