"""The native call of l2kv_paged_append_reserved: the same results as through ctypes, and what it does not take is left to the checks in Python."""
import pytest
import torch

import paper_2406_11430_amd as l2kv
from paper_2406_11430_amd import binding
from test_binding_calls_paged import append
from test_binding_calls_rows import Taken, ints


def test_what_is_not_a_device_tensor_is_left_to_the_checks():
    call = binding.calls().paged_append_reserved
    assert call() is None and call(*range(23)) is None
    assert call(*[None] * 22, binding._stream) is None
    assert call(*[torch.zeros((2, 2, 64))] * 22, binding._stream) is None


@pytest.mark.gpu
@pytest.mark.parametrize("without", [False, True])
def test_both_ways_are_the_same(without, monkeypatch):
    kw = dict(Q=None, Qr=None, q_weight=None, k_weight=None, lens_out=None, eps=0) if without else {}
    native, outputs = Taken(binding.calls()), []
    for calls in (native, binding._PythonCalls):
        monkeypatch.setattr(binding, "_calls", calls)
        a, outs = append(**kw)
        l2kv.l2kv_paged_append_reserved(**a, ends=None if without else ints(17, 6), stream=torch.cuda.current_stream())
        outputs.append([a[o].clone() for o in outs if a[o] is not None])
    assert native.count == 1
    for x, y in zip(*outputs):
        assert torch.equal(x, y) and x.abs().sum() > 0


@pytest.mark.gpu
@pytest.mark.parametrize("change", [lambda x: x.long(), lambda x: x[:-1].contiguous(), lambda x: x.cpu(), lambda x: x.float(), lambda x: 5])
def test_wrong_ends_are_refused(change):
    with pytest.raises((AssertionError, AttributeError, TypeError, ValueError)):
        l2kv.l2kv_paged_append_reserved(**append()[0], ends=change(ints(17, 6)))
