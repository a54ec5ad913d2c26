"""The norms between two blocks, forward and backward, against a float64 statement.

Tolerances.  Outputs in bf16 are off by half a step, 2^-8 of their size (2^-9 nearest; 2^-8 covers the values just above a power of two),
and by what fp32 loses on the way: a mean of d squares and a reciprocal root, products and one sum, each term good to
(log2 d + 10) 2^-24 < 2^-19 of its size.  x is compared with the norm of the h' that the call itself stored.  Sums over T tokens of fp32 terms:
2^-19 of the terms, and T 2^-24 for the additions, of the sum of the absolute values."""
import numpy as np
import pytest

import rows_plain as plain
from paper_2608_15241_b200 import workloads as wl

from gpu_util import Guarded, to_bits, to_dev

pytestmark = pytest.mark.gpu

EPS, SCALE = 1e-5, 0.7
HALF, FP32 = 2.0 ** -8, 2.0 ** -19


def _inputs(T, d, gate, post, seed=0):
    n = lambda k, std=1.0, shape=(T, d): wl.normal_bf16(seed * 100 + k, 1, shape, std)  # noqa: E731
    w = lambda k: plain.to_bf16(1 + 0.1 * np.random.default_rng(seed * 10 + k).standard_normal(d))  # noqa: E731
    i = dict(h=n(1), o=n(2, 3.0), dx=n(3, 0.1), dhn=n(4, 0.1), w_pre=w(1), w_post=w(2) if post else None, gate=None, gate_rows=None)
    i["h"][:, d // 3] = plain.to_bf16(np.array([40.0]))[0]              # a channel that is much larger than the others
    if gate == "shared":
        i["gate"] = n(5, 0.5, (d,))
    if gate == "rows":
        i["gate_rows"] = n(6, 0.5)
    return i


def _wide(i, k):
    return None if i[k] is None else plain.widen(i[k])


def _norm(i, d, eps=EPS):
    from paper_2608_15241_b200.binding import BlockNorm
    dev = {k: None if i[k] is None else to_dev(i[k]) for k in ("w_post", "w_pre", "gate")}
    return BlockNorm(d, scale=SCALE, eps=eps, **dev)


def _close(got, ref, size, half=HALF):
    bad = np.abs(got - ref) - (half * np.abs(ref) + FP32 * size)
    assert (bad <= 0).all(), (float(bad.max()), np.unravel_index(bad.argmax(), bad.shape))


SHAPES = [(1, 8), (1, 4096), (3, 40), (2, 16384), (5, 1032), (7, 2560), (150, 264), (300, 512), (149, 4096), (160, 8200), (33, 5120)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("gate,post", [("none", True), ("shared", True), ("rows", True), ("shared", False), ("none", False)])
def test_forward(T, d, gate, post):
    import torch
    i = _inputs(T, d, gate, post)
    gh, gx = Guarded(T * d * 2), Guarded(T * d * 2)
    g = i["gate_rows"]
    h_new, x = _norm(i, d).forward(to_dev(i["h"]), to_dev(i["o"]), gate_rows=None if g is None else to_dev(g),
                                   h_new=gh.view(torch.bfloat16, (T, d)), x=gx.view(torch.bfloat16, (T, d)))
    torch.cuda.synchronize()
    assert gh.intact() and gx.intact()
    h_new, x = plain.widen(to_bits(h_new)), plain.widen(to_bits(x))
    ref, size = plain.norm_h(_wide(i, "h"), _wide(i, "o"), _wide(i, "w_post"), _wide(i, "gate" if g is None else "gate_rows"), SCALE, EPS)
    _close(h_new, ref, size)
    want = plain.norm_x(h_new, plain.widen(i["w_pre"]), EPS)
    _close(x, want, np.abs(want))


@pytest.mark.parametrize("T,d", [(1, 4096), (40, 264), (300, 512), (200, 2560)])
@pytest.mark.parametrize("form", plain.FORMS)
def test_checkpoints_are_those_of_what_is_stored_and_x_is_the_norm_of_it(T, d, form):
    """One pass gives h', x and their checkpoints; a call on h' alone, and stores of h' and x, give the same bits."""
    import torch
    from paper_2608_15241_b200.binding import Checkpoint, checkpoint_store
    i = _inputs(T, d, "shared", True)
    norm = _norm(i, d)
    xk, hk = Checkpoint.empty(T, d, form), Checkpoint.empty(T, d, "int8")
    h_new, x = norm.forward(to_dev(i["h"]), to_dev(i["o"]), x_checkpoint=xk, h_checkpoint=hk)
    same, x_again = norm.forward(h_new)
    assert same is h_new and torch.equal(x, x_again)
    for kept, t, f in ((xk, x, form), (hk, h_new, "int8")):
        want = checkpoint_store(t, f)
        assert torch.equal(kept.data, want.data) and torch.equal(kept.scales, want.scales)


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("gate,post,form", [("shared", True, "bf16"), ("rows", True, "int8"), ("none", True, "e4m3"), ("shared", False, "int8"),
                                            ("none", False, "bf16")])
def test_backward(T, d, gate, post, form):
    import torch
    from paper_2608_15241_b200 import binding as b
    i = _inputs(T, d, gate, post)
    norm = _norm(i, d)
    keep = (lambda k: to_dev(i[k])) if form == "bf16" else (lambda k: b.checkpoint_store(to_dev(i[k]), form))
    g = i["gate_rows"]
    gs = Guarded(3 * d * 4)
    sums = gs.view(torch.float32, (3, d))
    sums.fill_(0.25)                                                    # they are added to
    gws = Guarded(b.lml_block_norm_workspace_bytes(0, T, d))
    gdh, gdo = Guarded(T * d * 2), Guarded(T * d * 2)
    dh, do, dgate = norm.backward(keep("h"), keep("o"), to_dev(i["dx"]), to_dev(i["dhn"]), gate_rows=None if g is None else to_dev(g),
                                  dh=gdh.view(torch.bfloat16, (T, d)), d_o=gdo.view(torch.bfloat16, (T, d)), dw_pre=sums[0],
                                  dw_post=sums[1] if post else None, dgate=sums[2] if gate == "shared" else None, workspace=gws.payload)
    torch.cuda.synchronize()
    assert gs.intact() and gws.intact() and gdh.intact() and gdo.intact()
    r = plain.norm_backward(plain.kept(i["h"], form), plain.kept(i["o"], form), _wide(i, "w_post"), _wide(i, "w_pre"),
                            _wide(i, "gate" if g is None else "gate_rows"), SCALE, EPS, _wide(i, "dx"), _wide(i, "dhn"))
    _close(plain.widen(to_bits(dh)), r["dh"], r["m_dh"])
    _close(plain.widen(to_bits(do)), r["do"], r["m_do"])
    if gate == "rows":
        _close(plain.widen(to_bits(dgate)), r["dgate_rows"], r["m_dgate_rows"])
    got = sums.cpu().numpy().astype(np.float64)
    for k, name, there in ((0, "dw_pre", True), (1, "dw_post", post), (2, "dgate", gate == "shared")):
        if there:
            assert (np.abs(got[k] - 0.25 - r[name]) <= (FP32 + T * 2.0 ** -24) * (r["m_" + name] + 0.25)).all(), name
        else:
            assert (got[k] == 0.25).all(), name


# More rows than a wave: two and four vectors per thread; the rings of the backward pass gone round many times, by one and by several groups of
# warps, of one stage (the widest row of all inputs), and by the kernels of the usual call, whose threads' columns make up the row.
@pytest.mark.parametrize("T,d", [(1300, 264), (2000, 2560), (6100, 264), (6100, 1032), (6100, 8)])
def test_forward_of_many_rows(T, d):
    test_forward(T, d, "shared", True)


@pytest.mark.parametrize("T,d,gate,form", [(2000, 264, "rows", "int8"), (900, 5120, "shared", "e4m3"), (1000, 4096, "shared", "int8"), (700, 1024, "none", "bf16"),
                                           (400, 6152, "rows", "e4m3"), (500, 8192, "shared", "bf16"), (400, 16384, "rows", "bf16"), (310, 16384, "none", "int8")])
def test_backward_of_many_rows(T, d, gate, form):
    test_backward(T, d, gate, True, form)


def test_backward_parts_that_are_not_there():
    """Only dx, only dh_new, frozen norms: what is left out changes nothing else; the same bits with and without the sums."""
    import torch
    T, d = 70, 520
    i = _inputs(T, d, "shared", True)
    norm = _norm(i, d)
    h, o, dx, dhn = (to_dev(i[k]) for k in ("h", "o", "dx", "dhn"))
    zero = torch.zeros_like(dx)
    sums = torch.zeros((3, d), device="cuda")
    full = norm.backward(h, o, dx, dhn, dw_pre=sums[0], dw_post=sums[1], dgate=sums[2])
    frozen = norm.backward(h, o, dx, dhn)
    assert torch.equal(full[0], frozen[0]) and torch.equal(full[1], frozen[1]) and frozen[2] is None
    for a, z in (((dx, None), (dx, zero)), ((None, dhn), (zero, dhn))):
        p, q = norm.backward(h, o, *a), norm.backward(h, o, *z)
        assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])
    dh, do, _ = norm.backward(None, o, None, dhn)
    assert torch.equal(dh, dhn) and torch.equal(do, norm.backward(h, o, zero, dhn)[1])
    dh, do, _ = norm.backward(h, None, dx, dhn)
    assert do is None and torch.equal(dh, full[0])


def test_outputs_in_the_place_of_inputs():
    import torch
    T, d = 90, 1032
    i = _inputs(T, d, "rows", True)
    norm = _norm(i, d)
    h, o, g = to_dev(i["h"]), to_dev(i["o"]), to_dev(i["gate_rows"])
    h_new, x = norm.forward(h, o, gate_rows=g)
    dx, dhn = to_dev(i["dx"]), to_dev(i["dhn"])
    dh, do, dg = norm.backward(h_new, o, dx, dhn, gate_rows=g)
    h2, o2 = h.clone(), o.clone()
    norm.forward(h2, o2, gate_rows=g, h_new=h2, x=o2)
    assert torch.equal(h2, h_new) and torch.equal(o2, x)
    dx2, dhn2 = dx.clone(), dhn.clone()
    _, _, dg2 = norm.backward(h_new, o, dx2, dhn2, gate_rows=g, dh=dhn2, d_o=dx2)
    assert torch.equal(dhn2, dh) and torch.equal(dx2, do) and torch.equal(dg2, dg)


def test_rows_are_on_their_own_and_not_finite_ones_stay_where_they_are():
    """A row of zeros, and rows with Inf or NaN, concern nobody else."""
    import torch
    T, d = 20, 264
    i = _inputs(T, d, "shared", True)
    norm = _norm(i, d)
    h, o = to_dev(i["h"]), to_dev(i["o"])
    h_new, x = norm.forward(h, o)
    h2, o2 = h.clone(), o.clone()
    o2[3], h2[7, 5], o2[11, 9] = 0.0, float("inf"), float("nan")
    hn2, x2 = norm.forward(h2, o2)
    assert torch.equal(hn2[3], h2[3])                                   # the norm of zeros is zero
    for t in range(T):
        if t not in (3, 7, 11):
            assert torch.equal(hn2[t], h_new[t]) and torch.equal(x2[t], x[t])
    assert torch.isnan(x2[11]).any() and torch.isinf(hn2[7, 5])
    alone = norm.forward(h[4:5].contiguous(), o[4:5].contiguous())
    size = x[4].float().abs().max()
    assert (alone[1][0].float() - x[4].float()).abs().max() <= 2.0 ** -7 * size


def test_captured_and_on_a_stream_of_its_own_and_twice_the_same():
    import torch
    T, d = 200, 2560
    i = _inputs(T, d, "shared", True)
    norm = _norm(i, d)
    h, o, dx, dhn = (to_dev(i[k]) for k in ("h", "o", "dx", "dhn"))
    sums = torch.zeros((3, d), device="cuda")
    want = norm.backward(h, o, dx, dhn, dw_pre=sums[0], dw_post=sums[1], dgate=sums[2])
    h_new, x = norm.forward(h, o)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    again = torch.zeros((3, d), device="cuda")
    torch.cuda.synchronize()
    h_s, x_s = norm.forward(h, o, stream=s)
    got = norm.backward(h, o, dx, dhn, dw_pre=again[0], dw_post=again[1], dgate=again[2], stream=s)
    s.synchronize()
    assert torch.equal(h_s, h_new) and torch.equal(x_s, x) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(again, sums)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again.zero_()
        h_g, x_g = norm.forward(h, o)
        got = norm.backward(h_g, o, dx, dhn, dw_pre=again[0], dw_post=again[1], dgate=again[2])
    o.copy_(to_dev(wl.normal_bf16(77, 1, (T, d), 1.0)))
    graph.replay()
    graph.replay()
    h_new, x = norm.forward(h, o)
    sums.zero_()
    want = norm.backward(h_new, o, dx, dhn, dw_pre=sums[0], dw_post=sums[1], dgate=sums[2])
    torch.cuda.synchronize()
    assert torch.equal(h_g, h_new) and torch.equal(x_g, x) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(again, sums)


def test_no_tokens():
    import torch
    i = _inputs(1, 64, "none", True)
    norm = _norm(i, 64)
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    sums = torch.ones(64, device="cuda")
    assert norm.forward(e, e)[0].shape == (0, 64)
    norm.backward(e, e, e, e, dw_pre=sums)
    assert (sums == 1).all()
