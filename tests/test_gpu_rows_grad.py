"""Adapter gradients with x as bf16 rows or an 8-bit checkpoint, against a float64 statement on the values that the rows stand for.

Tolerance.  u and v are fp32 and enter the second product as three bf16 values, which is all of them.  Sums of K and of T terms run in fp32: on the
tensor cores in steps of 16 that may each cut off a bit, at most 32 of them before the sum is taken out, and then in one rounded addition for
512 terms.  So min(K / 16, 32) + K / 512 steps of 2^-23, the same of T, and 32 for scale, split and the joining of parts, of the sum of the absolute
values of the terms.  The Frobenius error: 32 additions that lose half a unit of 2^-23 each, always towards zero, of partial sums that are half of the
whole on average, in either product: 2 * 32 * 2^-25 = 1.9e-6; held to 3e-6."""
import numpy as np
import pytest

import rows_plain as plain
from paper_2608_15241_b200 import workloads as wl

from gpu_util import Guarded, to_bits, to_dev

pytestmark = pytest.mark.gpu


class Case:
    """Two tables with the same adapters in different slots, a batch in segments."""

    def __init__(self, T, K, N, ranks, lengths, seg_entry, seed=1, scales=None, spare=2):
        import torch
        from paper_2608_15241_b200.binding import Table
        assert sum(lengths) == T
        self.T, self.K, self.N, self.ranks = T, K, N, ranks
        self.x, self.dy = wl.normal_bf16(seed, 1, (T, K), 1.0), wl.normal_bf16(seed, 2, (T, N), 0.05)
        self.A = [wl.normal_bf16(seed, 10 + i, (r, K), 0.05) for i, r in enumerate(ranks)]
        self.B = [wl.normal_bf16(seed, 50 + i, (N, r), 0.05) for i, r in enumerate(ranks)]
        self.scales = scales or [2.0 - 0.3 * i for i in range(len(ranks))]
        self.offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.seg_entry = list(seg_entry)
        self.t, self.tT = Table(K, N, len(ranks) + spare), Table(N, K, len(ranks) + spare)
        order = list(range(len(ranks)))
        slots, slots_T = {}, {}
        for e in order:
            slots[e] = self.t.register_adapter(e, 1, to_dev(self.A[e]), to_dev(self.B[e]), self.scales[e])
        for e in reversed(order):
            slots_T[e] = self.tT.register_adapter_transposed(e, 1, to_dev(self.A[e]), to_dev(self.B[e]), self.scales[e])
        self.slots, self.slots_T = slots, slots_T
        dev = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
        self.so = dev(self.offsets)
        self.ids, self.ids_T = dev([slots.get(e, -1) for e in seg_entry]), dev([slots_T.get(e, -1) for e in seg_entry])

    def rows(self, form):
        from paper_2608_15241_b200 import binding as b
        return to_dev(self.x) if form == "bf16" else b.checkpoint_store(to_dev(self.x), form)

    def buffers(self, fill=0.0):
        import torch
        gA, gB = Guarded(self.t.max_slots * 64 * self.K * 4), Guarded(self.t.max_slots * self.N * 64 * 4)
        dA, dB = gA.view(torch.float32, (self.t.max_slots, 64, self.K)), gB.view(torch.float32, (self.t.max_slots, self.N, 64))
        dA.fill_(fill)
        dB.fill_(fill)
        return gA, gB, dA, dB

    def run(self, form, accumulate=False, fill=0.0, x=None, dy=None, ids=None, ids_T=None, so=None, buffers=None):
        import torch
        from paper_2608_15241_b200 import binding as b
        gA, gB, dA, dB = buffers or self.buffers(fill)
        ws = Guarded(b.lml_backward_rows_workspace_bytes(self.t.handle, self.T, len(self.seg_entry)))
        self.t.backward_adapters_rows(self.tT, self.rows(form) if x is None else x, to_dev(self.dy) if dy is None else dy, self.so if so is None else so,
                                      self.ids if ids is None else ids, self.ids_T if ids_T is None else ids_T, dA, dB, accumulate=accumulate,
                                      workspace=ws.payload)
        torch.cuda.synchronize()
        assert gA.intact() and gB.intact() and ws.intact()
        return dA.cpu().numpy().astype(np.float64), dB.cpu().numpy().astype(np.float64)

    def check(self, dA, dB, form, base=0.0, written=True):
        """Rows j < rank of the adapters hold base + the gradients; everything else holds `base` as it was filled."""
        ents = [(r, s, plain.widen(A), plain.widen(B)) for r, s, A, B in zip(self.ranks, self.scales, self.A, self.B)]
        refs = plain.gradients(plain.kept(self.x, form), plain.widen(self.dy), ents, self.offsets, self.seg_entry)
        add = base if not written else 0.0
        steps = lambda n: min(n / 16, 32) + n / 512  # noqa: E731
        c = (steps(max(self.K, self.N)) + steps(self.T) + 32) * 2.0 ** -23
        for e, (rA, rB, mA, mB) in enumerate(refs):
            s, r = self.slots[e], self.ranks[e]
            gA, gB = dA[s, :r] - add, dB[s, :, :r] - add
            for got, ref, size in ((gA, rA, mA), (gB, rB, mB)):
                bad = np.abs(got - ref) - (c * size + 2.0 ** -23 * abs(add))
                assert (bad <= 0).all(), (e, float(bad.max()))
                if np.linalg.norm(ref) > 0 and not add:
                    assert np.linalg.norm(got - ref) <= 3e-6 * np.linalg.norm(ref), (e, np.linalg.norm(got - ref) / np.linalg.norm(ref))
            dA[s, :r], dB[s, :, :r] = base, base
        assert (dA == base).all() and (dB == base).all(), "rows behind the rank, or free slots, were written"

    def close(self):
        assert self.t.device_status() == 0 and self.tT.device_status() == 0
        self.t.close()
        self.tT.close()


CASES = [
    (1, 64, 64, [16], [1], [0]),
    (1, 4096, 264, [4], [1], [0]),
    (17, 72, 136, [1, 33], [9, 8], [1, 0]),
    (64, 128, 128, [16], [64], [0]),
    (65, 136, 520, [64], [65], [0]),
    (129, 200, 1032, [8, 16], [1, 128], [1, 0]),
    (300, 264, 136, [4, 16, 1, 33, 64], [40, 0, 100, 3, 57, 30, 70], [0, 1, 2, 3, -1, 4, 2]),
    (300, 1032, 200, [16, 16], [150, 150], [-1, -1]),
    (700, 1024, 512, [32], [700], [0]),
    (1100, 520, 264, [16, 48], [127, 129, 500, 344], [0, 1, 0, 1]),
    (2100, 256, 384, [16], [2000, 100], [0, -1]),
    (40, 5128, 8, [16], [40], [0]),                                    # sums that are taken out of the accumulators, steps of one half
    (3000, 264, 8, [64, 8], [2900, 100], [0, 1]),
    (257, 8, 328, [33], [257], [0]),
    (449, 712, 72, [16, 64], [192, 64, 65, 128], [0, 1, 0, 1]),
    (30, 544, 2056, [8, 16, 32, 64, 8, 16, 32], [1, 2, 1, 1, 0, 3, 1, 1, 1, 2, 1, 1, 2, 0, 1, 3, 1, 1, 1, 2, 1, 1, 1, 1], [k % 7 for k in range(24)]),
]


@pytest.mark.parametrize("form", ("int8", "e4m3", "bf16"))
@pytest.mark.parametrize("T,K,N,ranks,lengths,seg_entry", CASES)
def test_gradients(T, K, N, ranks, lengths, seg_entry, form):
    c = Case(T, K, N, ranks, lengths, seg_entry)
    c.check(*c.run(form, fill=0.5), form, base=0.5)
    c.close()


@pytest.mark.parametrize("T,lengths", [(1, [1, 0]), (10, [7, 3]), (70, [66, 4]), (137, [3, 134])])
@pytest.mark.parametrize("K", (368, 4096))
def test_scale_words_that_end_where_the_memory_ends(T, lengths, K):
    """A tile has 128 rows and the array of scale words ends with the last row of the batch; nothing behind it may be read."""
    import torch
    from paper_2608_15241_b200 import binding as b
    c = Case(T, K, 264, [16, 33], lengths, [0, 1])
    want = c.run("int8")
    kept = c.rows("int8")
    buffer = torch.empty(22 << 20, dtype=torch.uint8, device="cuda")          # a block of memory of its own, without a rest
    n, m = kept.scales.numel(), kept.data.numel()
    at = (buffer.numel() - n) // 16 * 16                                      # (both arrays are 16-byte aligned)
    scales, data = buffer[at:at + n].view(kept.scales.shape), buffer[:m].view(kept.data.shape)
    scales.copy_(kept.scales)
    data.copy_(kept.data)
    got = c.run("int8", x=b.Checkpoint(data, scales, K, "int8"))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    c.check(*got, "int8")
    c.close()


@pytest.mark.parametrize("form", ("int8", "bf16"))
def test_accumulated_over_batches_and_the_same_bits_again(form):
    c = Case(300, 264, 136, [4, 16, 33], [40, 0, 100, 3, 57, 100], [0, 1, 2, 1, -1, 0])
    first = c.run(form)
    b = c.buffers()
    one = c.run(form, accumulate=True, buffers=b)
    assert np.array_equal(first[0], one[0]) and np.array_equal(first[1], one[1])
    two = c.run(form, accumulate=True, buffers=b)
    assert np.array_equal(two[0], 2 * one[0]) and np.array_equal(two[1], 2 * one[1])
    dA, dB = c.run(form, accumulate=True, fill=0.25)
    c.check(dA, dB, form, base=0.25, written=False)
    c.close()


def test_many_segments():
    """More segments than a list holds, most of them shorter than a step of 16, of three adapters and of none."""
    rng = np.random.default_rng(2)
    lengths = rng.integers(0, 9, 450).tolist()
    seg = rng.integers(-1, 3, 450).tolist()
    c = Case(sum(lengths), 200, 136, [16, 5, 64], lengths, seg)
    for form in ("int8", "bf16"):
        c.check(*c.run(form), form)
    c.close()


def test_accumulate_false_writes_zeros_where_a_live_adapter_has_no_token():
    c = Case(40, 128, 72, [16, 20], [40], [0])
    dA, dB = c.run("int8", fill=3.0)
    s = c.slots[1]
    assert (dA[s, :20] == 0).all() and (dB[s, :, :20] == 0).all() and (dA[s, 20:] == 3).all()
    c.check(dA, dB, "int8", base=3.0)
    c.close()


def test_no_tokens():
    import torch
    from paper_2608_15241_b200 import binding as b
    c = Case(40, 128, 72, [16, 20], [40], [0])
    for accumulate, want in ((True, 3.0), (False, 0.0)):
        gA, gB, dA, dB = c.buffers(3.0)
        z = torch.zeros(2, dtype=torch.int32, device="cuda")
        b.lora_mixed_linear_backward_adapters_rows(c.t.handle, c.tT.handle, None, 0, 0, z.data_ptr(), z.data_ptr(), z.data_ptr(), 1,
                                                   dA.data_ptr(), dB.data_ptr(), accumulate, 0, 0, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert gA.intact() and gB.intact()
        for e, r in enumerate(c.ranks):
            assert (dA[c.slots[e], :r] == want).all() and (dB[c.slots[e], :, :r] == want).all() and (dA[c.slots[e], r:] == 3).all()
    c.close()


@pytest.mark.parametrize("form", ("int8", "bf16"))
def test_values_that_are_not_finite_reach_their_own_adapter_only(form):
    """Inf in x, NaN in dy and Inf in an adapter, at segment borders inside a tile and in its last step of 16."""
    lengths, seg = [37, 21, 70, 5, 60], [0, 1, 0, 1, 2]
    c = Case(sum(lengths), 136, 200, [16, 8, 12], lengths, seg)
    clean = c.run(form)
    x, dy = c.x.copy(), c.dy.copy()
    for t in (37, 57, 128, 132):                                        # first and last rows of adapter 1's segments
        x[t, 3], dy[t, 5] = 0x7F80, 0x7FC0
    c.x, c.dy = x, dy
    got = c.run(form)
    for e in (0, 2):
        s = c.slots[e]
        assert np.array_equal(got[0][s], clean[0][s]) and np.array_equal(got[1][s], clean[1][s])
    s = c.slots[1]
    assert np.isnan(got[0][s, :8]).any() and np.isnan(got[1][s, :, :8]).any()
    c.close()


def test_bindings_that_do_not_hold_together_add_nothing_and_raise_the_flag():
    import torch
    from paper_2608_15241_b200.binding import FLAG_BAD_OFFSETS, FLAG_BAD_SLOT
    c = Case(100, 136, 72, [16, 8], [30, 30, 40], [0, 1, -1])
    clean = c.run("int8")
    for place, value, t_flag, T_flag in (("ids", 3, FLAG_BAD_SLOT, FLAG_BAD_SLOT), ("ids", 99, FLAG_BAD_SLOT, FLAG_BAD_SLOT),
                                         ("ids_T", -1, 0, FLAG_BAD_SLOT), ("ids_T", c.slots_T[0], 0, FLAG_BAD_SLOT), ("ids", -7, FLAG_BAD_SLOT, FLAG_BAD_SLOT)):
        moved = getattr(c, place).clone()
        moved[1] = value
        dA, dB = c.run("int8", **{place: moved})
        assert (c.t.device_status(), c.tT.device_status()) == (t_flag, T_flag), (place, value)
        for e in range(2):
            s = c.slots[e]
            assert np.array_equal(dA[s], clean[0][s] * (e == 0)) and np.array_equal(dB[s], clean[1][s] * (e == 0))
    for bad in ([0, 30, 20, 100], [0, 30, 60, 99], [1, 30, 60, 100], [0, 30, 2000000000, 100], [0, -5, 60, 100]):
        dA, dB = c.run("int8", accumulate=True, fill=1.0, so=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        assert (dA == 1).all() and (dB == 1).all(), bad
        assert c.t.device_status() == FLAG_BAD_OFFSETS and c.tT.device_status() == 0
    c.close()


def test_refusals_of_a_live_table():
    import torch
    from paper_2608_15241_b200 import binding as b
    c = Case(40, 128, 72, [16], [40], [0])
    _, _, dA, dB = c.buffers()
    dy, kept = to_dev(c.dy), c.rows("int8")
    n = b.lml_backward_rows_workspace_bytes(c.t.handle, 40, 1)
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    other = b.Table(128, 128, 2)

    def call(tT=c.tT, rows=kept.rows, dyp=dy.data_ptr(), T=40, so=c.so.data_ptr(), G=1, dAp=dA.data_ptr(), wsp=ws.data_ptr(), wsn=n):
        b.lora_mixed_linear_backward_adapters_rows(c.t.handle, tT.handle, rows, dyp, T, so, c.ids.data_ptr(), c.ids_T.data_ptr(), G, dAp,
                                                   dB.data_ptr(), False, wsp, wsn, 0)
    bad_rows = b.Rows(kept.data.data_ptr(), 0, b.ROWS_INT8)
    for why, kw in ((b.ERR_INVALID_ARG, dict(tT=other)), (b.ERR_INVALID_ARG, dict(rows=None)), (b.ERR_INVALID_ARG, dict(rows=bad_rows)),
                    (b.ERR_INVALID_ARG, dict(rows=b.Rows(kept.data.data_ptr(), kept.scales.data_ptr(), 9))), (b.ERR_INVALID_ARG, dict(dyp=0)),
                    (b.ERR_INVALID_ARG, dict(dyp=dy.data_ptr() + 2)), (b.ERR_INVALID_ARG, dict(T=-1)), (b.ERR_INVALID_ARG, dict(G=0)),
                    (b.ERR_INVALID_ARG, dict(so=0)), (b.ERR_INVALID_ARG, dict(dAp=0)), (b.ERR_INVALID_ARG, dict(dAp=dA.data_ptr() + 4)),
                    (9, dict(wsn=n - 1)), (9, dict(wsp=0)), (9, dict(wsp=ws.data_ptr() + 16))):
        with pytest.raises(b.LmlError) as err:
            call(**kw)
        assert err.value.status == why, kw
    other.close()
    c.close()


def test_captured_and_on_a_stream_of_its_own():
    import torch
    c = Case(200, 264, 136, [16, 33], [90, 110], [0, 1])
    x, dy = c.rows("int8"), to_dev(c.dy)
    want = c.run("int8")
    s = torch.cuda.Stream()
    _, _, dA, dB = c.buffers()
    torch.cuda.synchronize()
    c.t.backward_adapters_rows(c.tT, x, dy, c.so, c.ids, c.ids_T, dA, dB, accumulate=False, stream=s)
    s.synchronize()
    assert np.array_equal(dA.cpu().numpy(), want[0]) and np.array_equal(dB.cpu().numpy(), want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.t.backward_adapters_rows(c.tT, x, dy, c.so, c.ids, c.ids_T, dA, dB, accumulate=False)
    c.dy = wl.normal_bf16(91, 2, (200, 136), 0.05)
    dy.copy_(to_dev(c.dy))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    got = dA.cpu().numpy().astype(np.float64), dB.cpu().numpy().astype(np.float64)
    want = c.run("int8")
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    c.close()


@pytest.mark.parametrize("form", ("int8", "bf16"))
def test_many_calls_back_to_back(form):
    """Long runs of whole units beside short ones, call after call without a pause: no role of a kernel may fall a turn of its ring behind."""
    import torch
    c = Case(1500, 1032, 4104, [16, 33], [900, 7, 593], [0, 1, 1])
    x, dy = c.rows(form), to_dev(c.dy)
    want = c.run(form)
    sets = [c.buffers() for _ in range(3)]
    for k in range(30):
        _, _, dA, dB = sets[k % 3]
        c.t.backward_adapters_rows(c.tT, x, dy, c.so, c.ids, c.ids_T, dA, dB, accumulate=False)
    torch.cuda.synchronize()
    for _, _, dA, dB in sets:
        assert np.array_equal(dA.cpu().numpy(), want[0]) and np.array_equal(dB.cpu().numpy(), want[1])
    c.check(*want, form)
    c.close()


def test_near_the_call_that_rounds_its_small_products():
    """lora_mixed_linear_backward_adapters on the same bf16 rows: its rounding of u and v, 2^-9 of every term, and no more."""
    import torch
    c = Case(300, 264, 136, [4, 16, 64], [100, 120, 80], [0, 1, 2])
    dA, dB = c.run("bf16")
    oA, oB = torch.zeros((c.t.max_slots, 64, c.K), device="cuda"), torch.zeros((c.t.max_slots, c.N, 64), device="cuda")
    c.t.backward_adapters(c.tT, to_dev(c.x), to_dev(c.dy), c.so, c.ids, c.ids_T, oA, oB)
    for got, old in ((dA, oA.cpu().numpy()), (dB, oB.cpu().numpy())):
        assert np.linalg.norm(got - old) <= 2.0 ** -8 * np.linalg.norm(got)
    c.close()
