"""Gradients from rows in tables that are full, adapters in the upper half of the slots among them; and calls on tables of their own at once."""
import numpy as np
import pytest

from gpu_util import to_dev
from test_gpu_rows_grad import Case

pytestmark = pytest.mark.gpu

FULL = 64


def _full(T, lengths, seg, ranks):
    return Case(T, 136, 200, ranks, lengths, seg, spare=0, scales=[1.0 + e / 64 for e in range(len(ranks))])


@pytest.mark.parametrize("form", ("int8", "e4m3", "bf16"))
def test_all_slots_of_a_full_table(form):
    """64 adapters; segments of the first, the last, and those on both sides of the middle, and of a few others, more than once."""
    ranks = [(1, 5, 16, 33, 64)[e % 5] for e in range(FULL)]
    seg = [0, 31, 32, 33, 63, 62, 31, 40, 63, 17, 32]
    lengths = [30, 129, 64, 1, 150, 16, 70, 3, 10, 128, 65]
    c = _full(sum(lengths), lengths, seg, ranks)
    assert sorted(c.slots.values()) == list(range(FULL))
    c.check(*c.run(form, fill=0.5), form, base=0.5)                     # the others' gradients are written, and zero
    dA, dB = c.run(form, accumulate=True, fill=0.25)
    c.check(dA, dB, form, base=0.25, written=False)
    c.close()


def test_only_slots_of_the_upper_half_are_left():
    ranks = [8] * FULL
    lengths, seg = [50, 90, 20], [40, 63, 32]
    c = _full(sum(lengths), lengths, seg, ranks)
    for e in range(FULL):
        if c.slots[e] < 32:
            c.t.retire_version(e, 1)
            c.tT.retire_version(e, 1)
    dA, dB = c.run("int8", fill=2.0)
    for e in range(FULL):                                               # free slots are left as they are
        s = c.slots[e]
        if s < 32:
            assert (dA[s] == 2).all() and (dB[s] == 2).all()
            dA[s, :8], dB[s, :, :8] = 0, 0
    c.check(dA, dB, "int8", base=2.0)
    c.close()


@pytest.mark.parametrize("form", ("e4m3", "bf16"))
def test_calls_on_two_pairs_of_tables_at_once(form):
    """Two streams, each with its own tables, buffers and workspaces, calls of different sizes queued on both: the bits of calls alone."""
    import torch
    cases = [Case(900, 1032, 520, [16, 33], [500, 400], [0, 1]), Case(333, 264, 2056, [64, 8, 16], [100, 33, 200], [0, 1, 2], seed=2)]
    want = [c.run(form) for c in cases]
    streams, sets = [torch.cuda.Stream() for _ in cases], []
    for c in cases:
        sets.append([(c.rows(form), to_dev(c.dy), *c.buffers()) for _ in range(2)])
    torch.cuda.synchronize()
    for k in range(20):
        for c, s, two in zip(cases, streams, sets):
            x, dy, _, _, dA, dB = two[k % 2]
            c.t.backward_adapters_rows(c.tT, x, dy, c.so, c.ids, c.ids_T, dA, dB, accumulate=False, stream=s)
    torch.cuda.synchronize()
    for c, two, (wA, wB) in zip(cases, sets, want):
        for _, _, gA, gB, dA, dB in two:
            assert gA.intact() and gB.intact()
            assert np.array_equal(dA.cpu().numpy(), wA) and np.array_equal(dB.cpu().numpy(), wB)
        c.close()


def test_nan_of_a_kept_block_stays_with_its_adapter():
    """E4M3 and INT8 blocks that held Inf or NaN read back as NaN: of that row's 32 columns, and in the gradients of that row's adapter only."""
    for form in ("e4m3", "int8"):
        lengths, seg = [37, 21, 70, 5, 60], [0, 1, 0, 1, 2]
        c = Case(sum(lengths), 136, 200, [16, 8, 12], lengths, seg)
        clean = c.run(form)
        x = c.x.copy()
        for t in (37, 57, 128, 132):                                    # first and last rows of adapter 1's segments
            x[t, 67] = 0x7F80
        c.x = x
        dA, dB = c.run(form)
        for e in (0, 2):
            s = c.slots[e]
            assert np.array_equal(dA[s], clean[0][s]) and np.array_equal(dB[s], clean[1][s])
        s = c.slots[1]
        assert np.isnan(dA[s, :8, 64:96]).all() and np.isfinite(dA[s, :8, :64]).all() and np.isfinite(dA[s, :8, 96:]).all()
        assert np.isnan(dB[s, :, :8]).all()                             # u of those tokens is NaN
        c.close()
