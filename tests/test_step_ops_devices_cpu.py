"""The batched serving step's operators refuse tensors, streams and rules that are not all on the current device, before any
allocation or launch: stand-ins for tensors of several GPUs, no GPU."""
import types

import pytest
import torch

from paper_2410_05165_gb300 import AtSpeedError, LogitRules, binding

I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
HERE, OTHER = torch.device("cuda", 0), torch.device("cuda", 1)


class Stand:
    """What the binding looks at of a contiguous tensor."""

    def __init__(self, shape, dtype, device=HERE):
        self.shape = torch.Size((shape,) if isinstance(shape, int) else shape)
        self.dtype, self.device, self.is_cuda = dtype, device, device.type == "cuda"

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Launched(Exception):
    pass


@pytest.fixture(autouse=True)
def library(monkeypatch):
    """A library that raises Launched for every entry point, and no GPU's memory."""
    class Lib:
        def __getattr__(self, name):
            if name == "atspeed_op_capture_id":
                return lambda stream: 0

            def entry(*args):
                raise Launched(name)
            return entry

    def outputs(device, stream, *specs):
        return [Stand(shape, dtype, device) for shape, dtype in specs]

    monkeypatch.setattr(binding, "load", Lib)
    monkeypatch.setattr(binding, "_outputs", outputs)
    monkeypatch.setattr(binding, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(binding, "op_tree_attention_workspace", lambda device, stream: Stand((4096,), torch.uint8))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)


def _plan(**kw):
    a = dict(q_len=Stand((2,), I32), kv_len=Stand((2,), I32), block_table=Stand((2, 4), I32), free=Stand((9,), I32),
             n_free=Stand((1,), I32), page_size=16, max_tokens=8, parent=Stand((8,), I32), mask_words=1)
    a.update(kw)
    return binding.op_batch_plan(**a)


def _append(**kw):
    a = dict(qkv=Stand((3, 512), F32), n_heads=4, kc=Stand((4, 16, 2, 64), BF16), vc=Stand((4, 16, 2, 64), BF16),
             slot=Stand((3,), torch.int64), pos=Stand((3,), I32))
    a.update(kw)
    return binding.op_rope_append(**a)


def _attention(**kw):
    a = dict(q=Stand((3, 4, 64), BF16), kc=Stand((4, 16, 2, 64), BF16), vc=Stand((4, 16, 2, 64), BF16), cu_q=Stand((2,), I32),
             ctx_len=Stand((1,), I32), block_table=Stand((1, 4), I32), mask=Stand((3, 1), I32), out=Stand((3, 4, 64), BF16),
             lse=Stand((3, 4), F32))
    a.update(kw)
    return binding.op_tree_attention(**a)


def _adjust(**kw):
    a = dict(logits=Stand((3, 100), F32), req=Stand((3,), I32), rules=LogitRules(temperature=Stand((2,), F32)),
             mask=Stand((3, 1), I32), state=Stand((3,), I32), out=Stand((3, 100), F32))
    a.update(kw)
    return binding.op_adjust_logits(**a)


CALLS = {"plan": (_plan, dict(q_len=((2,), I32), kv_len=((2,), I32), block_table=((2, 4), I32), free=((9,), I32),
                              n_free=((1,), I32), parent=((8,), I32))),
         "append": (_append, dict(qkv=((3, 512), F32), kc=((4, 16, 2, 64), BF16), vc=((4, 16, 2, 64), BF16),
                                  slot=((3,), torch.int64), pos=((3,), I32))),
         "attention": (_attention, dict(q=((3, 4, 64), BF16), kc=((4, 16, 2, 64), BF16), vc=((4, 16, 2, 64), BF16),
                                        cu_q=((2,), I32), ctx_len=((1,), I32), block_table=((1, 4), I32), mask=((3, 1), I32),
                                        out=((3, 4, 64), BF16), lse=((3, 4), F32))),
         "logits": (_adjust, dict(logits=((3, 100), F32), req=((3,), I32), mask=((3, 1), I32), state=((3,), I32),
                                  out=((3, 100), F32)))}


@pytest.mark.parametrize("op", CALLS)
def test_one_device_reaches_the_library(op):
    with pytest.raises(Launched):
        CALLS[op][0]()
    with pytest.raises(Launched):
        CALLS[op][0](stream=types.SimpleNamespace(device=HERE))


@pytest.mark.parametrize("op,arg", [(op, arg) for op in CALLS for arg in CALLS[op][1]])
@pytest.mark.parametrize("device", [OTHER, torch.device("cpu")])
def test_a_tensor_elsewhere_is_refused(op, arg, device):
    shape, dtype = CALLS[op][1][arg]
    with pytest.raises(AtSpeedError) as e:
        CALLS[op][0](**{arg: Stand(shape, dtype, device)})
    assert e.value.status == binding.E_ARG


@pytest.mark.parametrize("op", CALLS)
def test_tensors_of_a_device_that_is_not_current_are_refused(op, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(AtSpeedError) as e:
        CALLS[op][0]()
    assert e.value.status == binding.E_ARG


@pytest.mark.parametrize("op", CALLS)
def test_a_stream_of_another_device_is_refused(op):
    with pytest.raises(AtSpeedError) as e:
        CALLS[op][0](stream=types.SimpleNamespace(device=OTHER))
    assert e.value.status == binding.E_ARG


def test_rules_of_another_device_are_refused():
    for make in (lambda: LogitRules(temperature=Stand((2,), F32), frequency=Stand((2,), F32, OTHER)),
                 lambda: LogitRules(temperature=Stand((2,), F32, torch.device("cpu"))),
                 lambda: _adjust(rules=LogitRules(temperature=Stand((2,), F32, OTHER)))):
        with pytest.raises(AtSpeedError) as e:
            make()
        assert e.value.status == binding.E_ARG
    with pytest.raises(Launched):
        _adjust(rules=LogitRules(n_req=0))
