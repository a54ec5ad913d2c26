"""8-bit checkpoints on the GPU: data and scales byte for byte those of the plain statement, the loaded values exactly what they stand
for, nothing written outside the buffers."""
import numpy as np
import pytest

import rows_plain as plain
from paper_2608_15241_b200 import workloads as wl

from gpu_util import Guarded, to_bits, to_dev

pytestmark = pytest.mark.gpu


def _run(bits, form, device="cuda:0"):
    import torch
    from paper_2608_15241_b200 import binding as b
    T, d = bits.shape
    gd, gs, gx = (Guarded(n, device) for n in (b.lml_checkpoint_data_bytes(T, d), b.lml_checkpoint_scale_bytes(T, d), T * d * 2))
    kept = b.Checkpoint(gd.payload.view(T, -1), gs.payload.view(-1, T, 4), d, form)
    out = kept.store(to_dev(bits)).load(gx.view(torch.bfloat16, (T, d)))
    torch.cuda.synchronize()
    assert gd.intact() and gs.intact() and gx.intact()
    return kept.data.cpu().numpy(), kept.scales.cpu().numpy(), to_bits(out)


@pytest.mark.parametrize("form", plain.FORMS)
@pytest.mark.parametrize("T,d", [(1, 8), (1, 32), (3, 40), (2, 128), (5, 136), (7, 264), (2, 4104), (33, 512), (1, 11008)])
def test_store_and_load(T, d, form):
    bits = wl.normal_bf16(T * 7 + d, 1, (T, d), 1.0)
    bits[0, d // 2] = plain.to_bf16(np.array([37.25]))[0]               # an outlier
    data, scales = plain.encode(bits, form)
    got_data, got_scales, got = _run(bits, form)
    assert np.array_equal(got_scales, scales)
    assert np.array_equal(got_data, data)
    assert np.array_equal(plain.widen(got), plain.decode(data, scales, d, form))


@pytest.mark.parametrize("form", plain.FORMS)
def test_borders_of_the_formats(form):
    """Every bf16 value as the largest of a block, halves of a step, the smallest and the largest numbers."""
    pos = np.arange(0x0000, 0x7F80, 3, dtype=np.uint16)                 # finite, subnormals among them
    rng = np.random.default_rng(1)
    bits = np.zeros((len(pos), 32), np.uint16)
    bits[:, 0] = pos | 0x8000
    bits[:, 1] = pos
    # values of the same and of lower binades, all signs
    below = np.maximum(pos[:, None].astype(np.int64) - rng.integers(0, 0x500, (len(pos), 30)), 0).astype(np.uint16)
    bits[:, 2:] = below | (rng.integers(0, 2, below.shape).astype(np.uint16) << 15)
    data, scales = plain.encode(bits, form)
    got_data, got_scales, got = _run(bits, form)
    assert np.array_equal(got_scales, scales)
    assert np.array_equal(got_data, data)
    assert np.array_equal(plain.widen(got), plain.decode(data, scales, 32, form))


@pytest.mark.parametrize("form", plain.FORMS)
def test_blocks_that_are_not_finite_read_back_as_nan_and_leave_the_others_alone(form):
    bits = wl.normal_bf16(9, 1, (4, 104), 1.0)
    clean = bits.copy()
    bits[1, 33], bits[2, 103], bits[3, 0] = 0x7F80, 0x7FC1, 0xFF80      # Inf, NaN, -Inf
    _, scales = plain.encode(bits, form)
    _, got_scales, got = _run(bits, form)
    assert np.array_equal(got_scales, scales) and (got_scales == 255).sum() == 3
    want = plain.kept(clean, form)
    v = plain.widen(got)
    for t, k in ((1, 1), (2, 3), (3, 0)):
        assert np.isnan(v[t, 32 * k:min(32 * k + 32, 104)]).all()
        want[t, 32 * k:32 * k + 32] = np.nan
    assert np.array_equal(v, want, equal_nan=True)


def test_a_stream_of_its_own_and_a_captured_pass():
    import torch
    from paper_2608_15241_b200 import binding as b
    bits = wl.normal_bf16(4, 1, (50, 264), 1.0)
    x, out, kept = to_dev(bits), torch.empty((50, 264), dtype=torch.bfloat16, device="cuda"), b.Checkpoint.empty(50, 264, "int8")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    kept.store(x, stream=s)
    kept.load(out, stream=s)
    s.synchronize()
    assert np.array_equal(plain.widen(to_bits(out)), plain.kept(bits, "int8"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept.store(x)
        kept.load(out)
    other = wl.normal_bf16(5, 1, (50, 264), 3.0)
    x.copy_(to_dev(other))
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(plain.widen(to_bits(out)), plain.kept(other, "int8"))
