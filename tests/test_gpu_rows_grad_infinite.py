"""Infinities in x and dy, in the gradients from bf16 rows: sums whose terms of infinite size have one sign are that infinity, as in the
formula; NaN where the formula has NaN, and nowhere else."""
import numpy as np
import pytest

import rows_plain as plain
from gpu_util import to_dev
from test_gpu_rows_grad import Case

pytestmark = pytest.mark.gpu

INF, NINF = 0x7F80, 0xFF80


def _formula(c):
    ents = [(r, s, plain.widen(A), plain.widen(B)) for r, s, A, B in zip(c.ranks, c.scales, c.A, c.B)]
    with np.errstate(invalid="ignore"):
        return [g[:2] for g in plain.gradients(plain.widen(c.x), plain.widen(c.dy), ents, c.offsets, c.seg_entry)]


def _kind(v):
    """0 finite, 1 and -1 the infinities, 2 NaN."""
    return np.where(np.isnan(v), 2, np.where(np.isposinf(v), 1, np.where(np.isneginf(v), -1, 0)))


@pytest.mark.parametrize("T,lengths,seg", [(40, [40], [0]), (700, [200, 300, 200], [0, 1, 0])])
@pytest.mark.parametrize("where", ("x", "dy"))
def test_infinite_values(T, lengths, seg, where):
    c = Case(T, 264, 136, [16, 40], lengths, seg)
    bits = getattr(c, where).copy()
    bits[5, 3], bits[17, 130] = INF, NINF                               # two tokens of the first adapter, two columns
    setattr(c, where, bits)
    dA, dB = c.run("bf16")
    for e, (rA, rB) in enumerate(_formula(c)):
        s, r = c.slots[e], c.ranks[e]
        for got, ref in ((dA[s, :r], rA), (dB[s, :, :r], rB)):
            assert np.array_equal(_kind(got), _kind(ref)), (e, np.unique(_kind(ref) * 10 + _kind(got)))
            ok = np.isfinite(ref)
            assert ok.all() or e == 0
            np.testing.assert_allclose(got[ok], ref[ok], rtol=1e-3, atol=1e-3)
    if where == "x":
        assert np.isinf(dA[c.slots[0], :16, 3]).all() and np.isinf(dA[c.slots[0], :16, 130]).all()
    c.close()


def test_an_infinite_adapter_concerns_its_own_gradients_only():
    """An adapter that holds Inf beside others, its segments sharing tiles with theirs: the others keep their bits; ranks that are no multiple of
    16, so that its columns stand beside padded ones."""
    lengths, seg = [37, 21, 70, 5, 60], [0, 1, 0, 1, 2]
    c = Case(sum(lengths), 136, 200, [16, 5, 12], lengths, seg)
    x, kept = to_dev(c.x), {f: c.rows(f) for f in ("int8", "e4m3")}
    clean = {f: c.run(f, x=x if f == "bf16" else kept[f]) for f in ("bf16", "int8", "e4m3")}
    A, B = c.A[1].copy(), c.B[1].copy()
    A[2, 7], B[9, 3] = INF, NINF
    c.t.retire_version(1, 1)
    c.tT.retire_version(1, 1)
    assert c.t.register_adapter(1, 2, to_dev(A), to_dev(B), c.scales[1]) == c.slots[1]
    assert c.tT.register_adapter_transposed(1, 2, to_dev(A), to_dev(B), c.scales[1]) == c.slots_T[1]
    c.A[1], c.B[1] = A, B
    ref = _formula(c)[1]
    for f, was in clean.items():
        dA, dB = c.run(f, x=x if f == "bf16" else kept[f])
        for e in (0, 2):
            s = c.slots[e]
            assert np.array_equal(dA[s], was[0][s]) and np.array_equal(dB[s], was[1][s])
        s = c.slots[1]
        assert (dA[s, 5:] == 0).all() and (dB[s, :, 5:] == 0).all()
        # u's third column and v's fourth are infinite, the others as they were
        assert np.isfinite(dA[s, [0, 1, 2, 4]]).all() and not np.isfinite(dA[s, 3]).any()
        assert np.isfinite(dB[s][:, [0, 1, 3, 4]]).all() and not np.isfinite(dB[s, :, 2]).any()
        if f == "bf16":
            assert np.array_equal(_kind(dA[s, :5]), _kind(ref[0])) and np.array_equal(_kind(dB[s, :, :5]), _kind(ref[1]))
    c.close()
