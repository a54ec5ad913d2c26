"""Host-only checks of the binding's row calls: what they refuse before anything is allocated or launched."""
from types import SimpleNamespace

import pytest

from paper_2608_15241_b200 import binding


class OnDevice:
    """As much of a CUDA tensor as a call looks at before it refuses a stream."""
    is_cuda, shape = True, (4, 64)

    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


def _stream(index):
    import torch
    return SimpleNamespace(device=torch.device("cuda", index), device_index=index, cuda_stream=0x10)


def _calls():
    kept = binding.Checkpoint.__new__(binding.Checkpoint)
    kept.device = 0
    table = binding.Table.__new__(binding.Table)
    table.device, table.handle = 0, 0
    norm, t = binding.BlockNorm(64), OnDevice(0)
    yield "load", lambda s: kept.load(stream=s)
    yield "store", lambda s: binding.checkpoint_store(t, stream=s)
    yield "forward", lambda s: norm.forward(t, stream=s)
    yield "backward", lambda s: norm.backward(None, t, None, t, stream=s)
    yield "backward", lambda s: norm.backward(t, None, t, None, stream=s)
    yield "gradients", lambda s: table.backward_adapters_rows(None, t, t, None, None, None, None, None, stream=s)


@pytest.mark.parametrize("name,call", list(_calls()))
def test_a_stream_of_another_device_is_refused(name, call):
    with pytest.raises(AssertionError, match="stream"):
        call(_stream(1))


def test_a_norm_keeps_what_it_was_made_of():
    """Its descriptor holds the weights' addresses: a weight, a scale or an eps put in their place would be ignored, and the memory of the weight that
    it drops read all the same."""
    norm = binding.BlockNorm(64, scale=0.5, eps=1e-3)
    for name, value in (("w_post", OnDevice(0)), ("w_pre", OnDevice(0)), ("gate", OnDevice(0)), ("scale", 2.0), ("eps", 1e-6), ("d", 128)):
        with pytest.raises(AttributeError):
            setattr(norm, name, value)
    assert (norm.d, norm.scale, norm.eps, norm.w_post, norm.w_pre, norm.gate) == (64, 0.5, 1e-3, None, None, None)
    assert (norm.desc.d, norm.desc.scale) == (64, 0.5) and not norm.desc.w_pre


def test_widths_that_no_call_takes():
    for d in (0, -8, 12, 16392):
        with pytest.raises(AssertionError):
            binding.BlockNorm(d)
    assert binding.BlockNorm(binding.MAX_NORM_WIDTH).d == 16384


def test_what_a_checkpoint_takes():
    from paper_2608_15241_b200 import build
    build.build()
    for T, d in ((0, 8), (1, 8), (5, 4104), (300, 136), (8192, 11008)):
        kept = binding.Checkpoint.__new__(binding.Checkpoint)
        kept.tokens, kept.width = T, d
        assert kept.nbytes() == binding.lml_checkpoint_data_bytes(T, d) + binding.lml_checkpoint_scale_bytes(T, d)
