"""What the gradients from rows say about a batch when table t holds no adapter at all: a call whose segments name slots that are free, or
whose offsets are malformed, raises the flags that it raises beside a live adapter, and writes nothing."""
import pytest

from test_gpu_rows_grad import Case

pytestmark = pytest.mark.gpu


def _batch(G):
    """Three segments, or more than the library works on at a time."""
    return ([30, 30, 40], [0, 1, -1]) if G == 3 else ([1 + g % 2 for g in range(G)], [g % 3 - 1 for g in range(G)])


@pytest.mark.parametrize("G", (3, 450))
@pytest.mark.parametrize("accumulate", (False, True))
def test_a_table_whose_adapters_are_all_retired(G, accumulate):
    import torch
    from paper_2608_15241_b200.binding import FLAG_BAD_OFFSETS, FLAG_BAD_SLOT
    lengths, seg = _batch(G)
    c = Case(sum(lengths), 136, 72, [16, 8], lengths, seg)
    for e in range(2):
        c.t.retire_version(e, 1)

    def call(**changed):
        dA, dB = c.run("int8", accumulate=accumulate, fill=1.0, **changed)
        assert (dA == 1).all() and (dB == 1).all()
        return c.t.device_status(), c.tT.device_status()

    # the slots of t are free, those of t_T hold adapters: both ends of a binding are wrong
    assert call() == (FLAG_BAD_SLOT, FLAG_BAD_SLOT)
    # tokens without an adapter
    none = torch.full((G,), -1, dtype=torch.int32, device="cuda")
    assert call(ids=none, ids_T=none) == (0, 0)
    # only t_T is named
    assert call(ids=none) == (FLAG_BAD_SLOT, FLAG_BAD_SLOT)
    for place, value in ((0, 1), (1, -5), (G // 2, c.T + 1), (G, c.T - 1)):
        so = c.so.clone()
        so[place] = value
        assert call(so=so, ids=none, ids_T=none) == (FLAG_BAD_OFFSETS, 0), (place, value)
    # both tables empty
    for e in range(2):
        c.tT.retire_version(e, 1)
    assert call() == (FLAG_BAD_SLOT, 0)
    c.close()


def test_no_tokens_and_no_adapters():
    import torch
    from paper_2608_15241_b200 import binding as b
    t, tT = b.Table(136, 72, 2), b.Table(72, 136, 2)
    dA, dB = torch.ones((2, 64, 136), device="cuda"), torch.ones((2, 72, 64), device="cuda")
    for accumulate in (False, True):
        b.lora_mixed_linear_backward_adapters_rows(t.handle, tT.handle, None, 0, 0, 0, 0, 0, 1, dA.data_ptr(), dB.data_ptr(), accumulate, 0, 0,
                                                   torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert t.last_launch_count() == 0 and t.device_status() == 0 and tT.device_status() == 0
        assert (dA == 1).all() and (dB == 1).all()
    t.close()
    tT.close()


@pytest.mark.parametrize("place", (0, 1, 160, 319, 320, 321, 449, 450))
def test_malformed_offsets_of_many_segments_add_nothing_anywhere(place):
    """A batch of more segments than the library works on at a time, one offset of which is wrong: the slices before it add nothing either."""
    from paper_2608_15241_b200.binding import FLAG_BAD_OFFSETS
    lengths, seg = _batch(450)
    c = Case(sum(lengths), 136, 72, [16, 8], lengths, seg)
    so = c.so.clone()
    so[place] = {0: 2, 450: c.T - 1}.get(place, c.T + 1)
    dA, dB = c.run("bf16", accumulate=True, fill=1.0, so=so)
    assert (dA == 1).all() and (dB == 1).all()
    assert c.t.device_status() == FLAG_BAD_OFFSETS and c.tT.device_status() == 0
    dA, dB = c.run("bf16", fill=0.5)                                    # and the next call is as always
    c.check(dA, dB, "bf16", base=0.5)
    c.close()
