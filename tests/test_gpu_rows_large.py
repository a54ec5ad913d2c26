"""Row calls on buffers whose offsets pass 32 bits.  The rows of a large batch are those of a small one over and over, so that every repetition must
give what the first one gives, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu


def _repeated(t, T):
    return t.repeat((T + t.shape[0] - 1) // t.shape[0], 1)[:T].contiguous()


def _same_repetitions(got, n):
    """Whether all rows are those of the first n, n at a time."""
    import torch
    whole = got.shape[0] // n * n
    return torch.equal(got[:whole].view(-1, n, got.shape[1]), got[:n].expand(whole // n, n, got.shape[1])) and torch.equal(got[whole:], got[:got.shape[0] - whole])


def _free():
    import gc
    import torch
    gc.collect()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", ("int8", "e4m3"))
@pytest.mark.parametrize("T,d", [(70001, 65544), (3, 1 << 24), (130, 1 << 24), (4194304, 8)])
def test_checkpoints(T, d, form):
    import torch
    from paper_2608_15241_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(3)
    n = min(T, 101 if d < 1 << 20 else 2)
    few = torch.randn(n, d, generator=g, device="cuda").to(torch.bfloat16)
    want = b.checkpoint_store(few, form).load()
    x = _repeated(few, T)
    kept = b.checkpoint_store(x, form)
    assert _same_repetitions(kept.load(out=x), n) and torch.equal(x[:n], want)
    del x, kept
    _free()


@pytest.mark.parametrize("form", ("bf16", "int8"))
def test_norms(form):
    """8.6 GB a tensor; rows in checkpoints of more than 4 GB."""
    import torch
    from paper_2608_15241_b200 import binding as b
    T, d, n = 1050001, 4104, 1009
    g = torch.Generator(device="cuda").manual_seed(4)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    norm = b.BlockNorm(d, w_post=mk(d), w_pre=mk(d), gate=mk(d), scale=0.5)
    few_h, few_o = mk(n, d), mk(n, d)
    h, o = _repeated(few_h, T), _repeated(few_o, T)
    kx = b.Checkpoint.empty(T, d, "int8") if form != "bf16" else None
    _, x = norm.forward(h, o, h_new=h, x_checkpoint=kx)
    assert _same_repetitions(h, n) and _same_repetitions(x, n)
    if kx is not None:
        want = b.checkpoint_store(x[:n].contiguous(), "int8")
        assert torch.equal(kx.data[-(T % n):], want.data[:T % n]) and torch.equal(kx.scales[:, -(T % n):], want.scales[:, :T % n])
        kh, ko = b.checkpoint_store(h, "int8"), b.checkpoint_store(o, "int8")
    else:
        kh, ko = h, o
    del kx
    few_dx, few_dh = mk(n, d), mk(n, d)
    x.copy_(_repeated(few_dx, T))
    dh_new = _repeated(few_dh, T)
    sums = torch.zeros((3, d), device="cuda")
    dh, d_o, _ = norm.backward(kh, ko, x, dh_new, dh=dh_new, d_o=x, dw_pre=sums[0], dw_post=sums[1], dgate=sums[2])
    assert _same_repetitions(dh, n) and _same_repetitions(d_o, n)
    # the sums: T / n times those of the n rows, but for T 2^-24 of the terms' sizes (fp32 additions, as in the small cases)
    few = torch.zeros((3, d), device="cuda")
    rows = (lambda t: t) if form == "bf16" else (lambda t: b.checkpoint_store(t, "int8"))
    norm.backward(rows(h[:n].contiguous()), rows(o[:n].contiguous()), few_dx, few_dh, dw_pre=few[0], dw_post=few[1], dgate=few[2])
    rest = torch.zeros((3, d), device="cuda")
    m = T % n
    norm.backward(rows(h[:m].contiguous()), rows(o[:m].contiguous()), few_dx[:m].contiguous(), few_dh[:m].contiguous(), dw_pre=rest[0], dw_post=rest[1],
                  dgate=rest[2])
    size = torch.zeros(3, d, device="cuda", dtype=torch.float64)
    for t0 in range(n):                                                 # sums of the terms' absolute values, from calls of one row each
        one = torch.zeros((3, d), device="cuda")
        norm.backward(rows(h[t0:t0 + 1].contiguous()), rows(o[t0:t0 + 1].contiguous()), few_dx[t0:t0 + 1], few_dh[t0:t0 + 1], dw_pre=one[0], dw_post=one[1],
                      dgate=one[2])
        size += one.abs()
    want = few.double() * (T // n) + rest.double()
    assert ((sums.double() - want).abs() <= (2.0 ** -18 + T * 2.0 ** -24) * size * (T // n + 1)).all()
    del h, o, x, dh_new, kh, ko, dh, d_o
    _free()


def test_gradients():
    """x of 4.4 GB in 8 bits, two segments of one adapter that begin inside a tile."""
    import torch
    from paper_2608_15241_b200 import binding as b
    K, N, r, s = 8200, 72, 5, 2.0
    n, times = 1000, 537                                                # rows, repetitions
    T = n * times
    g = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda std, *shape: (std * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)  # noqa: E731
    A, B, few_x, few_dy = mk(0.05, r, K), mk(0.05, N, r), mk(1.0, n, K), mk(0.05, n, N)
    t, tT = b.Table(K, N, 2), b.Table(N, K, 2)
    ids = [t.register_adapter(0, 1, A, B, s), -1, 0]
    ids_T = [tT.register_adapter_transposed(0, 1, A, B, s), -1, 0]
    ids[2], ids_T[2] = ids[0], ids_T[0]
    cut = n * (times - 2) + 77                                          # the middle segment has no adapter: the last thousand rows of it do not count
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    so = dev([0, cut, cut + n, T])
    x, dy = _repeated(few_x, T), _repeated(few_dy, T)
    kept = b.checkpoint_store(x, "int8")
    few = b.checkpoint_store(few_x, "int8").load().double()
    del x
    dA, dB = torch.full((2, 64, K), 0.5, device="cuda"), torch.full((2, N, 64), 0.5, device="cuda")
    t.backward_adapters_rows(tT, kept, dy, so, dev(ids), dev(ids_T), dA, dB, accumulate=False)
    torch.cuda.synchronize()
    assert t.device_status() == 0 and tT.device_status() == 0
    # all repetitions but one of every row
    a, bb, d64 = A.double(), B.double(), few_dy.double()
    v, u = s * d64 @ bb, s * few @ a.T
    steps = lambda k: min(k / 16, 32) + k / 512  # noqa: E731
    c = (steps(K) + steps(T) + 32) * 2.0 ** -23                         # as in the gradients' own test
    mv, mu = s * d64.abs() @ bb.abs(), s * few.abs() @ a.abs().T
    for got, ref, size in ((dA[ids[0], :r], v.T @ few, mv.T @ few.abs()), (dB[ids[0], :, :r], d64.T @ u, d64.abs().T @ mu)):
        assert ((got.double() - (times - 1) * ref).abs() <= c * (times - 1) * size).all()
    assert (dA[ids[0], r:] == 0.5).all() and (dB[ids[0], :, r:] == 0.5).all() and (dA[1 - ids[0]] == 0.5).all() and (dB[1 - ids[0]] == 0.5).all()
    t.close()
    tT.close()
    del kept, dy
    _free()
