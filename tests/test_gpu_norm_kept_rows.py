"""The norms' forward pass of many and of wide rows with the checkpoints that it writes, and outputs of the backward pass that the C call alone can
leave out or place."""
import numpy as np
import pytest

import rows_plain as plain
from gpu_util import Guarded, to_bits, to_dev
from test_gpu_block_norm import EPS, SCALE, _close, _inputs, _norm, _wide

pytestmark = pytest.mark.gpu


# two and four vectors per thread, rows that end inside a thread's vectors, a warp's, a block of 32 columns
@pytest.mark.parametrize("form", plain.FORMS)
@pytest.mark.parametrize("T,d", [(6100, 1032), (6100, 4104), (6100, 2560), (6100, 520), (3, 16376), (200, 8200), (1300, 4104), (6100, 8)])
def test_checkpoints_of_many_and_of_wide_rows(T, d, form):
    """Byte for byte what a store makes of h' and x; nothing outside; h' and x the same with and without them."""
    import torch
    from paper_2608_15241_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(T + d)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    norm = b.BlockNorm(d, w_post=mk(d), w_pre=mk(d), gate=mk(d), scale=0.5)
    h, o = mk(T, d), mk(T, d)
    guards, kept = [], []
    for f in (form, "int8" if form == "e4m3" else "e4m3"):
        gd, gs = Guarded(b.lml_checkpoint_data_bytes(T, d)), Guarded(b.lml_checkpoint_scale_bytes(T, d))
        guards += [gd, gs]
        kept.append(b.Checkpoint(gd.payload.view(T, -1), gs.payload.view(-1, T, 4), d, f))
    h_new, x = norm.forward(h, o, x_checkpoint=kept[0], h_checkpoint=kept[1])
    torch.cuda.synchronize()
    assert all(q.intact() for q in guards)
    for k, t in zip(kept, (x, h_new)):
        want = b.checkpoint_store(t, k.form)
        assert torch.equal(k.data, want.data) and torch.equal(k.scales, want.scales)
    plain_h, plain_x = norm.forward(h, o)
    assert torch.equal(plain_h, h_new) and torch.equal(plain_x, x)
    _, alone = norm.forward(h_new, x_checkpoint=kept[1])                # a norm without a block before
    assert torch.equal(alone, x)
    want = b.checkpoint_store(x, kept[1].form)
    assert torch.equal(kept[1].data, want.data) and torch.equal(kept[1].scales, want.scales)


@pytest.mark.parametrize("T,d", [(1, 40), (5, 1032), (300, 264), (170, 5128), (160, 8200)])
def test_outputs_of_the_forward_call_one_at_a_time(T, d):
    import torch
    from paper_2608_15241_b200 import binding as b
    i = _inputs(T, d, "rows", True)
    norm, h, o, g = _norm(i, d), to_dev(i["h"]), to_dev(i["o"]), to_dev(i["gate_rows"])
    h_new, x = norm.forward(h, o, gate_rows=g)
    stream = torch.cuda.current_stream().cuda_stream
    for k in range(4):
        out = [Guarded(T * d * 2) if k == j else None for j in range(2)]
        kept = [b.Checkpoint.empty(T, d, "int8") if k == 2 + j else None for j in range(2)]
        at = [0 if q is None else q.payload.data_ptr() for q in out]
        b.lml_block_norm(0, norm.desc, T, h.data_ptr(), o.data_ptr(), g.data_ptr(), at[0], at[1], None if kept[0] is None else kept[0].rows,
                         None if kept[1] is None else kept[1].rows, stream)
        torch.cuda.synchronize()
        for q, want in zip(out, (h_new, x)):
            assert q is None or (q.intact() and torch.equal(q.view(torch.bfloat16, (T, d)), want))
        for q, want in zip(kept, (x, h_new)):
            assert q is None or torch.equal(q.data, b.checkpoint_store(want, "int8").data)


@pytest.mark.parametrize("T,d,form", [(1, 40, "bf16"), (37, 264, "int8"), (700, 1032, "e4m3"), (300, 5128, "bf16"), (170, 8200, "int8"), (1000, 2560, "int8")])
def test_outputs_of_the_backward_call_one_at_a_time(T, d, form):
    """Each output on its own has the bits that it has beside the others, the gradient of the gate rows between canaries; against float64."""
    import torch
    from paper_2608_15241_b200 import binding as b
    i = _inputs(T, d, "rows", True)
    norm, g = _norm(i, d), to_dev(i["gate_rows"])
    keep = (lambda k: to_dev(i[k])) if form == "bf16" else (lambda k: b.checkpoint_store(to_dev(i[k]), form))
    h, o, dx, dh_new = keep("h"), keep("o"), to_dev(i["dx"]), to_dev(i["dhn"])
    rows = [b._as_rows(t, (T, d), "rows", 0) for t in (h, o)]
    ws = Guarded(b.lml_block_norm_workspace_bytes(0, T, d))

    def call(wanted):
        sizes = {"dh": T * d * 2, "d_o": T * d * 2, "dw_pre": 4 * d, "dw_post": 4 * d, "dgate_rows": T * d * 2}
        out = {k: Guarded(n, fill=0) if k in wanted else None for k, n in sizes.items()}
        at = {k: 0 if q is None else q.payload.data_ptr() for k, q in out.items()}
        needs = "dw_pre" in wanted or "dw_post" in wanted
        b.lml_block_norm_backward(0, norm.desc, T, rows[0], rows[1], g.data_ptr(), dx.data_ptr(), dh_new.data_ptr(), at["dh"], at["d_o"], at["dw_pre"],
                                  at["dw_post"], 0, at["dgate_rows"], ws.payload.data_ptr() if needs else 0, ws.nbytes if needs else 0,
                                  torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert ws.intact() and all(q is None or q.intact() for q in out.values())
        return {k: q.payload.clone() for k, q in out.items() if q is not None}

    names = ("dh", "d_o", "dw_pre", "dw_post", "dgate_rows")
    whole = call(names)
    for k in names:
        assert torch.equal(call((k,))[k], whole[k]), k
    r = plain.norm_backward(plain.kept(i["h"], form), plain.kept(i["o"], form), _wide(i, "w_post"), _wide(i, "w_pre"), _wide(i, "gate_rows"), SCALE, EPS,
                            _wide(i, "dx"), _wide(i, "dhn"))
    for k, name in (("dh", "dh"), ("d_o", "do"), ("dgate_rows", "dgate_rows")):
        _close(plain.widen(to_bits(whole[k].view(torch.bfloat16).view(T, d))), r[name], r["m_" + name])
    for k in ("dw_pre", "dw_post"):
        got = whole[k].view(torch.float32).cpu().numpy().astype(np.float64)
        assert (np.abs(got - r[k]) <= (2.0 ** -19 + T * 2.0 ** -24) * r["m_" + k]).all()


def test_every_input_of_the_backward_call_as_an_output():
    """dh where h' is kept, d_o where o is, the gate rows' gradient in their place."""
    import torch
    T, d = 333, 1032
    i = _inputs(T, d, "rows", True)
    from paper_2608_15241_b200 import binding as b
    norm = _norm(i, d)
    h, o, g, dx, dh_new = (to_dev(i[k]) for k in ("h", "o", "gate_rows", "dx", "dhn"))
    want = norm.backward(h, o, dx, dh_new, gate_rows=g)
    b.lml_block_norm_backward(0, norm.desc, T, b.Rows(h.data_ptr(), None, b.ROWS_BF16), b.Rows(o.data_ptr(), None, b.ROWS_BF16), g.data_ptr(), dx.data_ptr(),
                              dh_new.data_ptr(), h.data_ptr(), o.data_ptr(), 0, 0, 0, g.data_ptr(), 0, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for got, ref in zip((h, o, g), want):
        assert torch.equal(got, ref)
