"""The row operators and the layer together, as a training step uses them: norm with checkpoints -> layer -> norm; then back, with
the adapter gradients and the norms' gradients taken from the checkpoints.  Compared with a float64 statement of the same step that takes over
the rounded values of the step between operators (so every operator is held to its own tolerance), and with differences of the loss."""
import numpy as np
import pytest

import rows_plain as plain
from paper_2608_15241_b200 import workloads as wl

from gpu_util import to_bits, to_dev

pytestmark = pytest.mark.gpu


def test_a_training_step_of_one_projection():
    import torch
    from paper_2608_15241_b200.binding import BlockNorm, Checkpoint, Table, checkpoint_store
    T, d, eps = 300, 264, 1e-5
    lengths, seg, ranks, s = [120, 40, 140], [0, 1, -1], [16, 8], 2.0
    bits = lambda k, shape, std: wl.normal_bf16(31, k, shape, std)  # noqa: E731
    h0, W0 = bits(1, (T, d), 1.0), bits(2, (d, d), 0.05)
    A, B = [bits(10 + i, (r, d), 0.05) for i, r in enumerate(ranks)], [bits(20 + i, (d, r), 0.05) for i, r in enumerate(ranks)]
    w1, w2, w3 = (plain.to_bf16(1 + 0.1 * np.random.default_rng(k).standard_normal(d)) for k in range(3))
    gate, g_h, g_x = bits(3, (d,), 0.5), bits(4, (T, d), 0.05), bits(5, (T, d), 0.05)
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)

    t, tT = Table(d, d, 2), Table(d, d, 2)
    for i in range(2):
        t.register_adapter(i, 1, to_dev(A[i]), to_dev(B[i]), s)
        tT.register_adapter_transposed(i, 1, to_dev(A[i]), to_dev(B[i]), s)
    so, ids = torch.from_numpy(offsets).cuda(), torch.tensor(seg, dtype=torch.int32, device="cuda")
    first, second = BlockNorm(d, w_pre=to_dev(w1), eps=eps), BlockNorm(d, w_post=to_dev(w2), w_pre=to_dev(w3), gate=to_dev(gate), scale=0.5, eps=eps)

    kx, kh, kh2 = Checkpoint.empty(T, d, "int8"), Checkpoint.empty(T, d, "int8"), Checkpoint.empty(T, d, "int8")
    _, x = first.forward(to_dev(h0), x_checkpoint=kx, h_checkpoint=kh)
    o = t.lora_mixed_linear(x, to_dev(W0), so, ids)
    ko = checkpoint_store(o, "int8")
    h1, x2 = second.forward(to_dev(h0), o, h_checkpoint=kh2)
    # back
    sums = torch.zeros((4, d), device="cuda")
    dh, do, _ = second.backward(kh2, ko, to_dev(g_x), to_dev(g_h), dw_pre=sums[0], dw_post=sums[1], dgate=sums[2])
    dA, dB = torch.zeros((2, 64, d), device="cuda"), torch.zeros((2, d, 64), device="cuda")
    t.backward_adapters_rows(tT, kx, do, so, ids, ids, dA, dB, accumulate=False)
    dx = tT.lora_mixed_linear(do, to_dev(np.ascontiguousarray(W0.T)), so, ids)
    dh0, _, _ = first.backward(kh, None, dx, dh, dw_pre=sums[3])
    torch.cuda.synchronize()
    assert t.device_status() == 0 and tT.device_status() == 0

    # the same step in float64, from the rounded values that the step itself kept
    W = plain.widen
    xr, orr = W(to_bits(x)), W(to_bits(o))
    y = xr @ W(W0).T
    for g, e in enumerate(seg):
        if e >= 0:
            r = slice(offsets[g], offsets[g + 1])
            y[r] += s * (xr[r] @ W(A[e]).T) @ W(B[e]).T
    assert np.linalg.norm(orr - y) <= 5e-3 * np.linalg.norm(y)
    kept = lambda v: plain.kept(v, "int8")  # noqa: E731
    ref = plain.norm_backward(kept(to_bits(h1)), kept(to_bits(o)), W(w2), W(w3), W(gate), 0.5, eps, W(g_x), W(g_h))
    rel = lambda got, want: np.linalg.norm(got - want) / np.linalg.norm(want)  # noqa: E731
    assert rel(W(to_bits(dh)), ref["dh"]) <= 2.0 ** -8 and rel(W(to_bits(do)), ref["do"]) <= 2.0 ** -8
    got = sums.cpu().numpy().astype(np.float64)
    for k, name in enumerate(("dw_pre", "dw_post", "dgate")):
        assert rel(got[k], ref[name]) <= 2e-5, name
    ents = [(r, s, W(a), W(b)) for r, a, b in zip(ranks, A, B)]
    for e, (rA, rB, _, _) in enumerate(plain.gradients(kept(to_bits(x)), W(to_bits(do)), ents, offsets, seg)):
        assert rel(dA[e, :ranks[e]].cpu().numpy(), rA) <= 2e-5 and rel(dB[e, :, :ranks[e]].cpu().numpy(), rB) <= 2e-5
    ref0 = plain.norm_backward(kept(h0), None, None, W(w1), None, 1.0, eps, W(to_bits(dx)), W(to_bits(dh)))
    assert rel(W(to_bits(dh0)), ref0["dh"]) <= 2.0 ** -8 and rel(got[3], ref0["dw_pre"]) <= 2e-5

    # what the checkpoints cost: the step's gradients against those at the unrounded activations, in float64 throughout.  A value of a block of
    # 32 normal ones is off by 1/128 of its largest's binade (2 of their standard deviation, mostly): 2^-6 / sqrt(12) = 0.5 % rms of the rows
    exact = plain.gradients(xr, W(to_bits(do)), ents, offsets, seg)
    for e in range(2):
        assert rel(dA[e, :ranks[e]].cpu().numpy(), exact[e][0]) <= 2.0 ** -6 and rel(dB[e, :, :ranks[e]].cpu().numpy(), exact[e][1]) <= 2.0 ** -6
    t.close()
    tT.close()


def test_memory_of_calls_on_a_stream_that_is_behind():
    """Calls on a stream of their own that has other work to do first; meanwhile the current stream asks for memory and writes to it."""
    import torch
    from paper_2608_15241_b200.binding import BlockNorm, Table, checkpoint_store
    T, d, r = 300, 512, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    norm = BlockNorm(d, w_post=mk(d), w_pre=mk(d), gate=mk(d), scale=0.5)
    h, o, dx, dh = (mk(T, d) for _ in range(4))
    t, tT = Table(d, d, 2), Table(d, d, 2)
    A, B = mk(r, d), mk(d, r)
    ids, ids_T = t.register_adapter(0, 1, A, B, 1.0), tT.register_adapter_transposed(0, 1, A, B, 1.0)
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    so, ids, ids_T = dev([0, T]), dev([ids]), dev([ids_T])

    def step(stream):
        sums = torch.zeros((3, d), device="cuda")
        dA, dB = torch.zeros((2, 64, d), device="cuda"), torch.zeros((2, d, 64), device="cuda")
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
        h_new, x = norm.forward(h, o, stream=stream)
        kept = checkpoint_store(x, "int8", stream=stream)
        back = kept.load(stream=stream)
        gh, go, _ = norm.backward(h_new, o, dx, dh, dw_pre=sums[0], dw_post=sums[1], dgate=sums[2], stream=stream)
        t.backward_adapters_rows(tT, kept, dh, so, ids, ids_T, dA, dB, accumulate=False, stream=stream)
        junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << k for k in range(9, 24)) for _ in range(3)]
        torch.cuda.synchronize()
        del junk
        return h_new, x, back, gh, go, sums, dA, dB

    want, got = step(None), step(torch.cuda.Stream())
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    t.close()
    tT.close()
