"""The native calls of rotary positions, prompt and tree attention and accepted paths: the same results as through ctypes, and what
they do not take is left to the checks in Python."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding

NAMES = {"rotary_append": 18, "prompt_attn": 12, "tree_attn": 15, "append_path": 16}
DEV = "cuda"


def test_what_is_not_a_device_tensor_is_left_to_the_checks():
    native = binding.calls()
    for name, n in NAMES.items():
        call = getattr(native, name)
        assert call() is None and call(*range(n)) is None
        assert call(*[None] * (n - 1), binding._stream) is None
        assert call(*[torch.zeros((2, 2, 64))] * (n - 1), binding._stream) is None


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def longs(*v):
    return torch.tensor(v, dtype=torch.int64, device=DEV)


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def rotary(**kw):
    rows = torch.zeros((2, 40, 64), dtype=torch.bfloat16, device=DEV)
    qkv = rand(0, 5, 8, 64)
    a = dict(Q=qkv[:, :4], K=qkv[:, 4:6], V=qkv[:, 6:], positions=ints(1, 2, 3, 4, 5), freqs=l2kv.l2kv_rotary_freqs(32, 10000.0).to(DEV),
             Qr=torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=DEV), Kc=rows, Vc=rows.clone(), norms_c=torch.zeros((2, 40), device=DEV),
             pos_c=torch.zeros((2, 40), dtype=torch.int32, device=DEV), token_offsets=longs(0, 2, 5), slot_offsets=longs(0, 20, 40),
             lens_in=ints(3, 0), lens_out=ints(0, 0), layout=1, amplitude=1.5)
    a.update(kw)
    return a, ("Qr", "Kc", "Vc", "norms_c", "pos_c", "lens_out")


def prompt(**kw):
    a = dict(Q=rand(0, 9, 8, 64)[:, :4], K=rand(1, 2, 30, 64), V=rand(2, 2, 30, 64), q_offsets=longs(0, 4, 9), kv_offsets=longs(0, 10, 30),
             kv_lens=ints(8, 20), max_kv=20, O=torch.zeros((9, 4, 64), dtype=torch.bfloat16, device=DEV), workspace=None, scale=0.3)
    a.update(kw)
    return a, ("O",)


def tree(**kw):
    a = dict(Q=rand(0, 6, 8, 64)[:, :4], Kc=rand(1, 2, 30, 64), Vc=rand(2, 2, 30, 64), lens=ints(8, 15), slot_offsets=longs(0, 10, 30), max_len=15,
             Kt=rand(3, 2, 6, 64), Vt=rand(4, 2, 6, 64), node_offsets=longs(0, 2, 6), mask=ints(1, 3, 1, 3, 5, 11).view(6, 1),
             O=torch.zeros((6, 4, 64), dtype=torch.bfloat16, device=DEV), workspace=None, scale=0.0)
    a.update(kw)
    return a, ("O",)


def path(**kw):
    a = dict(Kt=rand(0, 2, 6, 64), Vt=rand(1, 2, 6, 64), norms_t=rand(2, 2, 6).float(), pos_t=ints(*range(12)).view(2, 6), node_offsets=longs(0, 2, 6),
             path=ints(0, 1, 2, 0, 1, 3).view(2, 3), path_lens=ints(2, 3), slot_offsets=longs(0, 10, 30), lens_in=ints(3, 5), lens_out=ints(0, 0),
             Kc=torch.zeros((2, 30, 64), dtype=torch.bfloat16, device=DEV), Vc=torch.zeros((2, 30, 64), dtype=torch.bfloat16, device=DEV),
             norms_c=torch.zeros((2, 30), device=DEV), pos_c=torch.zeros((2, 30), dtype=torch.int32, device=DEV))
    a.update(kw)
    return a, ("lens_out", "Kc", "Vc", "norms_c", "pos_c")


CALLS = {"rotary_append": (rotary, l2kv.l2kv_rotary_append), "prompt_attn": (prompt, l2kv.l2kv_prompt_attn),
         "tree_attn": (tree, l2kv.l2kv_tree_attn), "append_path": (path, l2kv.l2kv_stream_append_path)}


class Taken:
    """The native calls, which have to take what is passed on to them."""
    def __init__(self, native):
        self.native, self.count = native, 0

    def __getattr__(self, name):
        def call(*args):
            st = getattr(self.native, name)(*args)
            assert st is not None
            self.count += 1
            return st
        return call


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("without", [False, True])
def test_both_ways_are_the_same(name, without, monkeypatch):
    build, entry = CALLS[name]
    kw = {}
    if without:
        kw = {"rotary_append": dict(Q=None, Qr=None, token_offsets=None, slot_offsets=None, lens_in=None, lens_out=None,
                                    **{k: torch.zeros((2, 5, 64), dtype=torch.bfloat16, device=DEV) for k in ("Kc", "Vc")},
                                    norms_c=torch.zeros((2, 5), device=DEV), pos_c=torch.zeros((2, 5), dtype=torch.int32, device=DEV)),
              "prompt_attn": dict(kv_lens=None, scale=0, workspace=torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)),
              "tree_attn": dict(Kc=rand(1, 2, 2, 10, 64), Vc=rand(2, 2, 2, 10, 64), slot_offsets=longs(0, 20, 30), lens=ints(8, 10)),
              "append_path": {}}[name]
    native, outputs = Taken(binding.calls()), []
    for calls in (native, binding._PythonCalls):
        monkeypatch.setattr(binding, "_calls", calls)
        a, outs = build(**{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
        entry(**a, stream=torch.cuda.current_stream())
        outputs.append([a[o].clone() for o in outs if a[o] is not None])
    assert native.count == 1
    for x, y in zip(*outputs):
        assert torch.equal(x, y) and x.abs().sum() > 0


WRONG = [(name, key, change) for name, (build, _) in CALLS.items() for key, change in {
    "rotary_append": [("Q", "half"), ("K", "heads"), ("V", "float"), ("positions", "long"), ("freqs", "float"), ("Qr", "short"), ("Kc", "short"),
                      ("Vc", "half"), ("norms_c", "short"), ("pos_c", "long"), ("token_offsets", "int"), ("slot_offsets", "short"),
                      ("lens_in", "short"), ("lens_out", "long"), ("K", "cpu"), ("Kc", "turned")],
    "prompt_attn": [("Q", "half"), ("Q", "heads"), ("K", "float"), ("V", "short"), ("q_offsets", "int"), ("kv_offsets", "short"), ("kv_lens", "long"),
                    ("O", "float"), ("O", "short"), ("V", "cpu"), ("K", "turned")],
    "tree_attn": [("Q", "heads"), ("Kc", "float"), ("Vc", "short"), ("lens", "long"), ("lens", "short"), ("slot_offsets", "short"), ("Kt", "short"), ("Vt", "float"),
                  ("node_offsets", "int"), ("mask", "long"), ("mask", "short"), ("O", "float"), ("mask", "cpu"), ("Kt", "turned")],
    "append_path": [("Kt", "half"), ("Vt", "float"), ("norms_t", "half"), ("pos_t", "long"), ("node_offsets", "short"), ("path", "long"), ("path_lens", "short"),
                    ("slot_offsets", "int"), ("lens_in", "short"), ("lens_out", "long"), ("Kc", "short"), ("Vc", "short"), ("norms_c", "short"), ("pos_c", "long"),
                    ("Kc", "cpu"), ("Kt", "turned")]}[name]]


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
