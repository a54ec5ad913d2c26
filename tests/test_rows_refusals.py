"""Host-only checks of the row calls (checkpoints, block norms, gradients from rows): what they refuse before touching CUDA, and the
plain statements that the GPU tests compare with, on hand-worked values and against the rounding that a checkpoint promises."""
import ctypes

import numpy as np
import pytest

import rows_plain as plain
from paper_2608_15241_b200 import binding, build, workloads as wl

INVALID, CUDA, WORKSPACE = 1, 7, 9


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def P(n=16):
    """An aligned pointer that is never followed."""
    return ctypes.c_void_p(0x10000 + n * 256)


def rows(fmt=binding.ROWS_INT8, data=0x20000, scales=0x30000):
    return ctypes.byref(binding.Rows(data, scales, fmt))


def test_sizes(lib):
    assert lib.lml_checkpoint_data_bytes(3, 40) == 3 * 64 and lib.lml_checkpoint_scale_bytes(3, 40) == 3 * 4
    assert lib.lml_checkpoint_data_bytes(5, 4104) == 5 * 4128 and lib.lml_checkpoint_scale_bytes(5, 4104) == 5 * 33 * 4
    for T, d in ((-1, 64), (4, 0), (4, 12), (4, -8), (1 << 30, 64)):
        assert lib.lml_checkpoint_data_bytes(T, d) == 0 and lib.lml_checkpoint_scale_bytes(T, d) == 0
    assert lib.lml_backward_rows_workspace_bytes(None, 4, 1) == 0
    assert lib.lml_block_norm_workspace_bytes(0, -1, 64) == 0 and lib.lml_block_norm_workspace_bytes(0, 4, 16392) == 0


def test_checkpoint_refusals(lib):
    for call in (lambda dev, x, T, d, r: lib.lml_checkpoint_store(dev, x, T, d, r, None), lambda dev, x, T, d, r: lib.lml_checkpoint_load(dev, r, T, d, x, None)):
        assert call(0, P(), 0, 64, rows()) == 0                         # nothing to do
        assert call(-1, P(), 4, 64, rows()) == INVALID
        assert call(0, None, 4, 64, rows()) == INVALID
        assert call(0, ctypes.c_void_p(0x10008), 4, 64, rows()) == INVALID
        assert call(0, P(), -1, 64, rows()) == INVALID
        assert call(0, P(), 4, 60, rows()) == INVALID
        assert call(0, P(), 4, 64, None) == INVALID
        assert call(0, P(), 4, 64, rows(binding.ROWS_BF16)) == INVALID  # not a checkpoint
        assert call(0, P(), 4, 64, rows(3)) == INVALID
        assert call(0, P(), 4, 64, rows(data=0)) == INVALID
        assert call(0, P(), 4, 64, rows(scales=0)) == INVALID
        assert call(0, P(), 4, 64, rows(data=0x20008)) == INVALID
        assert call(0, P(), 4, 64, rows(scales=0x30004)) == INVALID


def desc(d=64, eps=1e-5, scale=1.0, w_post=0x1000, w_pre=0x2000, gate=0x3000):
    return ctypes.byref(binding.BlockNormDesc(d, eps, scale, w_post, w_pre, gate))


def test_block_norm_refusals(lib):
    def call(dev=0, p=None, T=4, h=P(1), o=P(2), gate_rows=None, h_new=P(3), x=P(4), xk=None, hk=None):
        return lib.lml_block_norm(dev, p or desc(), T, h, o, gate_rows, h_new, x, xk, hk, None)
    assert call(T=0) == 0
    assert lib.lml_block_norm(0, None, 4, P(), None, None, None, P(), None, None, None) == INVALID
    for bad in (dict(dev=-1), dict(T=-1), dict(h=None), dict(h=ctypes.c_void_p(0x10002)), dict(x=ctypes.c_void_p(0x10008)),
                dict(p=desc(d=60)), dict(p=desc(d=0)), dict(p=desc(d=16392)), dict(p=desc(eps=0.0)), dict(p=desc(eps=-1.0)),
                dict(p=desc(eps=float("nan"))), dict(p=desc(scale=float("nan"))), dict(p=desc(w_pre=0x2004)),
                dict(o=None),                                           # h_new without a block's output
                dict(gate_rows=P(5)),                                   # two gates
                dict(p=desc(w_pre=0)),                                  # x without its weights
                dict(h_new=None, x=None),                               # nothing to do
                dict(xk=rows(binding.ROWS_BF16)), dict(hk=rows(7)), dict(hk=rows(scales=0))):
        assert call(**bad) == INVALID, bad
    assert call(o=None, h_new=None, gate_rows=P(5), p=desc(gate=0)) == INVALID


def test_block_norm_backward_refusals(lib):
    def call(dev=0, p=None, T=4, h=rows(), o=rows(), gate_rows=None, dx=P(1), dhn=P(2), dh=P(3), do=P(4), dwpre=None, dwpost=None, dgate=None, dgr=None,
             ws=None, n=0):
        return lib.lml_block_norm_backward(dev, p or desc(), T, h, o, gate_rows, dx, dhn, dh, do, dwpre, dwpost, dgate, dgr, ws, n, None)
    assert call(T=0) == 0
    for bad in (dict(dev=-1), dict(T=-1), dict(p=desc(d=12)), dict(dx=None, dhn=None), dict(h=None), dict(h=rows(5)), dict(o=rows(data=0)),
                dict(p=desc(w_pre=0)), dict(o=None), dict(o=None, do=None, dwpost=P(6)), dict(o=None, do=None, dgate=P(6)),
                dict(dx=None, dwpre=P(6)), dict(p=desc(w_post=0), dwpost=P(6)), dict(p=desc(gate=0), dgate=P(6)), dict(dgr=P(6)),
                dict(gate_rows=P(7)), dict(dh=None, do=None), dict(dx=ctypes.c_void_p(0x10004)), dict(dwpre=ctypes.c_void_p(0x10004))):
        assert call(**bad) == INVALID, bad


def test_gradient_refusals(lib):
    assert lib.lora_mixed_linear_backward_adapters_rows(None, None, rows(), P(), 4, P(), P(), P(), 1, P(), P(), 1, P(), 0, None) == INVALID


def test_calls_without_a_gpu_fail_cleanly(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("has a GPU")
    assert lib.lml_checkpoint_store(0, P(), 4, 64, rows(), None) == CUDA
    assert lib.lml_block_norm(0, desc(), 4, P(1), P(2), None, P(3), P(4), None, None, None) == CUDA
    assert lib.lml_block_norm_backward(0, desc(), 4, rows(), rows(), None, P(1), P(2), P(3), P(4), None, None, None, None, None, 0, None) == CUDA
    assert lib.lml_block_norm_workspace_bytes(0, 4, 64) == 0


def test_the_plain_checkpoint_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [1.9921875, -1.0, 0.0078125, 0.0234375]                 # binade 0: steps of 1/64; the largest is 127.5 steps, clamped
    x[0, 32:34] = [-3.0, 0.046875]                                     # binade 1: steps of 1/32: -96 and 1.5, to even
    data, scales = plain.encode(plain.to_bf16(x), "int8")
    assert data.view(np.int8)[0, :4].tolist() == [127, -64, 0, 2] and data.view(np.int8)[0, 32:34].tolist() == [-96, 2]
    assert scales.shape == (1, 1, 4) and scales[0, 0].tolist() == [121, 122, 0, 0]
    data, scales = plain.encode(plain.to_bf16(x), "e4m3")
    v = plain.decode(data, scales, 40, "e4m3")
    # 1.9921875 > 448/256: the unit is 1/128, so 255 -> 256 (four significant bits)
    assert scales[0, 0].tolist() == [120, 120, 0, 0]
    assert v[0, 0] == 2.0 and v[0, 1] == -1.0 and v[0, 2] == 0.0078125 and v[0, 32] == -3.0


@pytest.mark.parametrize("form", plain.FORMS)
def test_the_plain_checkpoint_is_off_by_half_a_step(form):
    bits = wl.normal_bf16(5, 1, (16, 72), 1.0)
    x = plain.widen(bits)
    data, scales = plain.encode(bits, form)
    v = plain.decode(data, scales, 72, form)
    assert np.array_equal(plain.widen(plain.to_bf16(v)), v)             # exact in bf16
    step = 2.0 ** (np.repeat(scales.transpose(1, 0, 2).reshape(16, -1)[:, :3], 32, 1)[:, :72] - 127.0)
    bound = 0.5 * step if form == "int8" else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)
    assert (np.abs(v - x) <= bound).all()


def test_the_plain_norm_gradients_are_differences():
    rng = np.random.default_rng(3)
    T, d, eps, scale = 3, 24, 1e-3, 0.7
    h, o, dx, dhn = (rng.standard_normal((T, d)) for _ in range(4))
    w_post, w_pre, gate = (1 + 0.1 * rng.standard_normal(d) for _ in range(3))

    def loss(h, o, w_post, w_pre, gate):
        hn, _ = plain.norm_h(h, o, w_post, gate, scale, eps)
        return (plain.norm_x(hn, w_pre, eps) * dx).sum() + (hn * dhn).sum()

    hn, _ = plain.norm_h(h, o, w_post, gate, scale, eps)
    r = plain.norm_backward(hn, o, w_post, w_pre, gate, scale, eps, dx, dhn)
    args = [h, o, w_post, w_pre, gate]
    for i, name in enumerate(("dh", "do", "dw_post", "dw_pre", "dgate")):
        num = np.zeros_like(args[i])
        for k in np.ndindex(num.shape):
            two = []
            for s in (1e-6, -1e-6):
                moved = [a.copy() for a in args]
                moved[i][k] += s
                two.append(loss(*moved))
            num[k] = (two[0] - two[1]) / 2e-6
        assert np.abs(num - r[name]).max() < 1e-7, name
