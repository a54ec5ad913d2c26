"""What surrounds the layer in a training step, and in a decode step, as cases whose time and results can be compared:
the norms between two blocks, the 8-bit checkpoints of activations, and the adapter gradients taken from a checkpoint.

A case:
  kind      norm      forward: the norm of a block's output, its gate, the residual sum and the next block's norm
            back      its backward pass
            keep      a checkpoint of activations is stored, and later loaded
            grads     dA and dB of one projection, x kept as a checkpoint
  tokens, width       rows and columns (grads: width is d_in, out is d_out)
  form      none, int8, e4m3: how activations are kept (norm: x is written as a checkpoint too; back: o and the residual
            stream are checkpoints; grads: x is one)
  gate      none, shared (a value per channel) or rows (a row of values per token)
  post      whether the block's output has a norm of its own
  adapters, ranks, none, runs   grads: adapters, their ranks in turn, the share of tokens without one, and of how many
            requests (runs of tokens on one adapter) the batch consists

The plain forms are in 32 bits.  A checkpoint is 8-bit values [T][width up to a multiple of 32] and, per row and 32
columns, a power of two 2^(b - 127): bytes b in [128-column group][T][4].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-5
RESIDUAL = 0.7     # the residual scale
SCALE = 2.0        # of the adapters
FORMS = {"int8": (6, 0), "e4m3": (8, 3)}   # exponent of the largest value's binade, least scale byte


def _case(name, kind, tokens, width, form="none", gate="none", post=False, out=0, adapters=0, ranks="", none=0.0, runs=0):
    return dict(name=name, kind=kind, tokens=tokens, width=width, form=form, gate=gate, post=post, out=out, adapters=adapters,
                ranks=ranks, none=none, runs=runs)


def listed():
    return [
        # one agent generating alone: latency between two blocks of a decode step
        _case("norm_1", "norm", 1, 4096, gate="shared", post=True),
        # a crowded decode step of a wider model; the gate comes from the token
        _case("norm_40_rows", "norm", 40, 5120, gate="rows", post=True),
        # a training batch: the next projections' x is kept as a checkpoint from the same pass
        _case("norm_1000_int8", "norm", 1000, 4096, form="int8", gate="shared", post=True),
        # the largest prefill batch, a model with a pre-norm only
        _case("norm_8192", "norm", 8192, 4096),
        # a short training sequence of a small model, activations kept as they are
        _case("back_37_rows", "back", 37, 2560, gate="rows", post=True),
        # the training batch's way back, from checkpoints
        _case("back_1000_int8", "back", 1000, 4096, form="int8", gate="shared", post=True),
        # the largest batch, gated, from checkpoints with a wider range
        _case("back_8192_e4m3", "back", 8192, 5120, form="e4m3", gate="shared", post=True),
        # an odd width: blocks of 32 that end inside the row
        _case("keep_200_odd", "keep", 200, 4104, form="e4m3"),
        # an MLP's inner activations of the largest batch
        _case("keep_8192", "keep", 8192, 11008, form="int8"),
        # a short training batch of one adapter: latency
        _case("grads_100", "grads", 100, 4096, form="int8", out=4096, adapters=1, ranks="16", runs=1),
        # a background training batch of two adapters, gate / up
        _case("grads_1000", "grads", 1000, 4096, form="int8", out=11008, adapters=2, ranks="16", runs=4),
        # the largest batch, adapters of every rank, some tokens on the bare base, down
        _case("grads_8192_mixed", "grads", 8192, 11008, form="e4m3", out=4096, adapters=8, ranks="8,16,32,64", none=0.1, runs=24),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "back", "back", "keep", "grads", "grads", "grads"])
    form = rng.choice(["int8", "e4m3"]) if kind in ("keep", "grads") else rng.choice(["none", "none", "int8", "e4m3"])
    if kind == "grads":
        d_in, d_out = 8 * _log_int(rng, 16, 1376), 8 * _log_int(rng, 16, 1376)
        ranks = rng.choice(["16", "16", "8", "32", "8,16,32,64", "4,8,8", "1,5,33"])
        most = 8192 * (11008 + 2 * 4096) / (d_in + 2 * d_out)          # costs no more than the largest listed case
        tokens = _log_int(rng, 1, min(8192, int(most)))
        case = _case("", kind, tokens, d_in, form=form, out=d_out, adapters=rng.randint(1, 8), ranks=ranks,
                     none=rng.choice([0.0, 0.0, 0.1]), runs=rng.choice([1, 4, 9, 24]))
    else:
        width = 8 * (_log_int(rng, 8, 1376) if kind == "keep" else _log_int(rng, 32, 640))
        case = _case("", kind, _log_int(rng, 1, 8192), width, form=form)
        if kind != "keep":
            case["gate"] = rng.choice(["none", "shared", "rows"])
            case["post"] = case["gate"] != "none" or rng.random() < 0.5
    del case["name"]
    return case


def _block(case):
    """Whether a norm case has a block's output to add to the residual stream."""
    return case["post"] or case["gate"] != "none"


def _ranks(case):
    r = [int(v) for v in case["ranks"].split(",")]
    return [r[a % len(r)] for a in range(case["adapters"])]


def work(case):
    T, d = case["tokens"], case["width"]
    kept = T * d + T * math.ceil(d / 32)                               # a checkpoint
    rows = 2.0 * T * d
    act = rows if case["form"] == "none" else kept
    if case["kind"] == "keep":
        return {"bytes": 2 * rows + 2 * kept, "flops": 4.0 * T * d}
    if case["kind"] == "grads":
        n, ranks = case["out"], _ranks(case)
        mean = sum(ranks) / len(ranks) * (1 - case["none"])
        used = sum(ranks)
        return {"bytes": kept + 2.0 * T * n + 2.0 * used * (d + n) + 4.0 * used * (d + n), "flops": 2 * 2.0 * T * mean * (d + n)}
    block, gate = _block(case), {"none": 0.0, "shared": 2.0 * d, "rows": rows}[case["gate"]]
    vectors = 2.0 * d * (1 + case["post"])
    if case["kind"] == "norm":
        total = rows * (4 if block else 2) + gate + vectors            # h, o in; h', x out
        total += 2 * kept + rows if case["form"] != "none" else 0      # the checkpoint out, and its values
        return {"bytes": total, "flops": 14.0 * T * d}
    total = act * (2 if block else 1) + 3 * rows + vectors + 4.0 * d * (1 + case["post"])   # o, h', dx, dh' in; dh out
    total += (rows if block else 0) + gate * (2 if case["gate"] == "rows" else 3)
    return {"bytes": total, "flops": 30.0 * T * d}


# ---- state --------------------------------------------------------------------------------------------

def _pow2(e):
    """2^e in 32 bits, e an integer tensor from -127 (a subnormal) on."""
    half = torch.div(e, 2, rounding_mode="floor")
    return torch.exp2(half.float()) * torch.exp2((e - half).float())


def _encode(x, form):
    """A checkpoint of x: (values [T][width up to 32], scale bytes [groups of 128 columns][T][4])."""
    T, d = x.shape
    top, least = FORMS[form]
    v = torch.nn.functional.pad(x.float(), (0, -d % 32)).view(T, -1, 32)
    amax = v.abs().amax(2)
    m, e = torch.frexp(amax)                                           # amax = m 2^e, m in [0.5, 1)
    e = e - 1 - top + ((m > 0.875).int() if form == "e4m3" else 0)
    e = torch.where(amax > 0, e, -127).clamp(min=least - 127)
    q = v * _pow2(-e)[..., None]
    q = q.round().clamp(-127, 127).to(torch.int8).view(torch.uint8) if form == "int8" else q.to(torch.float8_e4m3fn).view(torch.uint8)
    b = torch.where(amax.isfinite(), e + 127, 255).to(torch.uint8)
    b = torch.nn.functional.pad(b, (0, -b.shape[1] % 4)).view(T, -1, 4).transpose(0, 1).contiguous()
    return q.view(T, -1), b


def _decode(kept, form, d):
    q, b = kept
    T = q.shape[0]
    v = (q.view(torch.int8) if form == "int8" else q.view(torch.float8_e4m3fn)).float().view(T, -1, 32)
    s = _pow2(b.transpose(0, 1).reshape(T, -1)[:, :v.shape[1]].int() - 127)
    return (v * s[..., None]).view(T, -1)[:, :d]


class _Inputs:
    """Everything that a case draws from its seed."""

    def __init__(self, case, seed):
        gen = torch.Generator(device="cuda").manual_seed(int(seed))

        def normal(*shape, std=1.0, mean=0.0):
            return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(torch.bfloat16)

        def activations(*shape):
            """A residual stream has a few channels that are much larger than the others."""
            big = torch.rand(shape[-1], generator=gen, device="cuda") < 0.01
            return (torch.randn(shape, generator=gen, device="cuda") * torch.where(big, 12.0, 1.0)).to(torch.bfloat16)

        T, d = case["tokens"], case["width"]
        if case["kind"] == "keep":
            self.x = activations(T, d)
        elif case["kind"] == "grads":
            n, ranks = case["out"], _ranks(case)
            self.x, self.dy = activations(T, d), normal(T, n, std=0.01)
            self.A = [normal(r, d, std=0.02) for r in ranks]
            self.B = [normal(n, r, std=0.02) for r in ranks]
            r = np.random.Generator(np.random.Philox(key=[int(seed), 1]))
            runs = min(case["runs"], T)
            cuts = np.sort(r.choice(np.arange(1, T), size=runs - 1, replace=False)) if runs > 1 else np.array([], int)
            self.offsets = np.concatenate([[0], cuts, [T]]).astype(np.int32)
            self.adapter = np.where(r.random(runs) < case["none"], -1, r.integers(0, case["adapters"], runs)).astype(np.int32)
        else:
            self.h, self.w_pre = activations(T, d), normal(d, std=0.1, mean=1.0)
            self.o = normal(T, d) if _block(case) else None
            self.w_post = normal(d, std=0.1, mean=1.0) if case["post"] else None
            self.gate = {"none": lambda: None, "shared": lambda: normal(d, std=0.2, mean=0.5),
                         "rows": lambda: normal(T, d, std=0.2, mean=0.5)}[case["gate"]]()
            if case["kind"] == "back":
                self.dx, self.dh_new = normal(T, d, std=0.01), normal(T, d, std=0.01)


def prepare(case, seed):
    """The inputs, what is kept from the forward pass, and the handles that a program keeps (norm weights, tables)."""
    i, form = _Inputs(case, seed), case["form"]
    state = dict(case=case, i=i)
    if case["kind"] == "back":
        keep = (lambda v: v) if form == "none" else (lambda v: _encode(v, form))
        state["h_new"], state["o"] = keep(i.h), None if i.o is None else keep(i.o)
    if case["kind"] == "grads":
        ranks = _ranks(case)
        state["x"] = _encode(i.x, form)
        state["A"] = torch.stack([torch.nn.functional.pad(A, (0, 0, 0, 64 - r)) for A, r in zip(i.A, ranks)])    # [adapter][64][d_in]
        state["B"] = torch.stack([torch.nn.functional.pad(B, (0, 64 - r)) for B, r in zip(i.B, ranks)])          # [adapter][d_out][64]
        state["offsets"], state["slots"] = torch.from_numpy(i.offsets).cuda(), torch.from_numpy(i.adapter).cuda()
        state["token_slot"] = torch.from_numpy(np.repeat(i.adapter, np.diff(i.offsets))).cuda()
    if own:
        from paper_2608_15241_b200 import binding
        if case["kind"] == "grads":
            d, n = case["width"], case["out"]
            state["table"], state["table_T"] = (binding.Table(a, b, max_slots=case["adapters"]) for a, b in ((d, n), (n, d)))
            for a, (A, B) in enumerate(zip(i.A, i.B)):                 # the registrations fill the slots in order
                state["table"].register_adapter(a, 1, A, B, SCALE)
                state["table_T"].register_adapter_transposed(a, 1, A, B, SCALE)
            state["dA"] = torch.zeros((case["adapters"], 64, d), dtype=torch.float32, device="cuda")
            state["dB"] = torch.zeros((case["adapters"], n, 64), dtype=torch.float32, device="cuda")
        elif case["kind"] != "keep":
            state["norm"] = binding.BlockNorm(case["width"], w_post=i.w_post, w_pre=i.w_pre, scale=RESIDUAL, eps=EPS,
                                              gate=i.gate if case["gate"] == "shared" else None)
    return state


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    return {"norm": _norm, "back": _back, "keep": _keep, "grads": _grads}[state["case"]["kind"]](state)


def _norm(state):
    case, i = state["case"], state["i"]
    form = case["form"]
    if own:
        from paper_2608_15241_b200 import binding
        kept = None if form == "none" else binding.Checkpoint.empty(case["tokens"], case["width"], form)
        h_new, x = state["norm"].forward(i.h, i.o, gate_rows=i.gate if case["gate"] == "rows" else None, x_checkpoint=kept)
        return [h_new, x] if kept is None else [h_new, x, kept.load()]
    h, x = i.h, i.h.float()
    if i.o is not None:
        n = i.o.float()
        if case["post"]:
            n = n * torch.rsqrt(n.square().mean(1, keepdim=True) + EPS) * i.w_post.float()
        if i.gate is not None:
            n = n * i.gate.float()
        h = (x + RESIDUAL * n).to(torch.bfloat16)                      # the residual stream is kept in bf16, and normed as it is kept
        x = h.float()
    x = (x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * i.w_pre.float()).to(torch.bfloat16)
    return [h, x] if form == "none" else [h, x, _decode(_encode(x, form), form, case["width"]).to(torch.bfloat16)]


def _back(state):
    """dh, do and the gradients of the norms' weights and of the gate (what there is of them)."""
    case, i = state["case"], state["i"]
    form, d = case["form"], case["width"]
    if own:
        from paper_2608_15241_b200 import binding
        wrap = (lambda v: v) if form == "none" else (lambda v: None if v is None else binding.Checkpoint(*v, width=d, form=form))
        sums = torch.zeros((3, d), dtype=torch.float32, device="cuda")
        rows = i.gate if case["gate"] == "rows" else None
        dh, do, dgate = state["norm"].backward(wrap(state["h_new"]), wrap(state["o"]), i.dx, i.dh_new, gate_rows=rows, dw_pre=sums[0],
                                               dw_post=sums[1] if case["post"] else None, dgate=sums[2] if case["gate"] == "shared" else None)
        got = [dh, sums[0], do, sums[1] if case["post"] else None, dgate]
        return [v for v in got if v is not None]
    values = (lambda v: v.float()) if form == "none" else (lambda v: _decode(v, form, d))
    h, dx = values(state["h_new"]), i.dx.float()
    rho = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    h = h * rho
    g = dx * i.w_pre.float()
    D = i.dh_new.float() + rho * (g - h * (g * h).mean(1, keepdim=True))
    out = [D.to(torch.bfloat16), (dx * h).sum(0)]
    if i.o is not None:
        o = values(state["o"])
        dn = RESIDUAL * D
        gated = dn if i.gate is None else dn * i.gate.float()
        if case["post"]:
            r = torch.rsqrt(o.square().mean(1, keepdim=True) + EPS)
            o = o * r
            g = gated * i.w_post.float()
            out += [(r * (g - o * (g * o).mean(1, keepdim=True))).to(torch.bfloat16), (gated * o).sum(0)]
            o = o * i.w_post.float()
        else:
            out += [gated.to(torch.bfloat16)]
        if i.gate is not None:
            out.append((dn * o).to(torch.bfloat16) if case["gate"] == "rows" else (dn * o).sum(0))
    return out


def _keep(state):
    x, form = state["i"].x, state["case"]["form"]
    if own:
        from paper_2608_15241_b200 import binding
        return binding.checkpoint_store(x, form).load()
    return _decode(_encode(x, form), form, x.shape[1]).to(torch.bfloat16)


def _grads(state):
    case, i = state["case"], state["i"]
    if own:
        from paper_2608_15241_b200 import binding
        x = binding.Checkpoint(*state["x"], width=case["width"], form=case["form"])
        state["table"].backward_adapters_rows(state["table_T"], x, i.dy, state["offsets"], state["slots"], state["slots"],
                                              state["dA"], state["dB"], accumulate=False)
        return [state["dA"], state["dB"]]
    T, S = case["tokens"], case["adapters"]
    x, dy = _decode(state["x"], case["form"], case["width"]), i.dy.float()
    A, B = state["A"].float(), state["B"].float()
    bound = (torch.arange(S, device="cuda") == state["token_slot"][:, None]).float()[..., None]                  # [T][adapter][1]
    u = SCALE * bound * (x @ A.view(S * 64, -1).t()).view(T, S, 64)
    v = SCALE * bound * (dy @ B.transpose(1, 2).reshape(S * 64, -1).t()).view(T, S, 64)
    dA = (v.view(T, -1).t() @ x).view(S, 64, -1)
    dB = (u.view(T, -1).t() @ dy).view(S, 64, -1).transpose(1, 2)
    return [dA, dB.contiguous()]


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _binade(a):
    """floor(log2 a), a > 0, where the logarithm of a power of two may come out just below it."""
    p = torch.floor(torch.log2(a))
    return p + (torch.exp2(p + 1) <= a).double()


def _kept64(x, form):
    """What a checkpoint of the bf16 rows x stands for."""
    T, d = x.shape
    v = torch.zeros((T, -(-d // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :d] = x.double()
    v = v.view(T, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    power = _binade(torch.where(top > 0, top, 1.0))
    if form == "int8":                                                 # steps of 2^-6 of the largest value's binade, 127 at most
        step = torch.exp2(power - 6)
        r = torch.clamp(torch.round(v / step), -127, 127) * step
    else:                                                              # four significant bits down to 2^-6, steps of 2^-9 below that
        unit = torch.exp2(power - 8)
        unit = torch.where(top > 448 * unit, 2 * unit, unit)
        a = v / unit
        step = torch.exp2(_binade(torch.clamp(a.abs(), min=2.0 ** -6)) - 3)
        r = torch.round(a / step) * step * unit
    return r.view(T, -1)[:, :d]


def exact(case, seed):
    i, form, kind = _Inputs(case, seed), case["form"], case["kind"]
    if kind == "keep":
        return _kept64(i.x, form)
    if kind == "grads":
        x, dy = _kept64(i.x, form), i.dy.double()
        dA = torch.zeros((case["adapters"], 64, x.shape[1]), dtype=torch.float64, device="cuda")
        dB = torch.zeros((case["adapters"], dy.shape[1], 64), dtype=torch.float64, device="cuda")
        for g, a in enumerate(i.adapter):
            if a >= 0:
                A, B, r = i.A[a].double(), i.B[a].double(), i.A[a].shape[0]
                xs, ds = x[i.offsets[g]:i.offsets[g + 1]], dy[i.offsets[g]:i.offsets[g + 1]]
                dA[a, :r] += SCALE * (ds @ B).t() @ xs
                dB[a, :, :r] += SCALE * ds.t() @ (xs @ A.t())
        return [dA, dB]
    d, wide = case["width"], lambda t: t.double()  # noqa: E731
    inv = lambda t: ((t * t).sum(1) / d + EPS).sqrt().reciprocal()[:, None]  # noqa: E731
    w, gate = wide(i.w_pre), 1.0 if i.gate is None else wide(i.gate)
    w_post = wide(i.w_post) if case["post"] else 1.0
    if kind == "norm":
        h = wide(i.h)
        if i.o is not None:
            o = wide(i.o)
            n = o * inv(o) * w_post if case["post"] else o
            h = wide((h + RESIDUAL * gate * n).to(torch.bfloat16))     # (kept in bf16, and normed as it is kept)
        x = h * inv(h) * w
        return [h, x] if form == "none" else [h, x, _kept64(x.to(torch.bfloat16), form)]
    h = wide(i.h) if form == "none" else _kept64(i.h, form)
    dx = wide(i.dx)
    s = inv(h)
    # x_j = h_j s w_j with s = (sum h^2 / d + eps)^(-1/2):  dL/dh_k = s w_k dx_k - s^3 h_k / d sum_j dx_j w_j h_j
    D = wide(i.dh_new) + s * w * dx - s ** 3 * h / d * (dx * w * h).sum(1, keepdim=True)
    out = [D, (dx * h * s).sum(0)]
    if i.o is not None:
        o = wide(i.o) if form == "none" else _kept64(i.o, form)
        dn = RESIDUAL * gate * D
        n = o
        if case["post"]:
            s = inv(o)
            n = o * s * w_post
            out += [s * w_post * dn - s ** 3 * o / d * (dn * w_post * o).sum(1, keepdim=True), (dn * o * s).sum(0)]
        else:
            out += [dn]
        if case["gate"] != "none":
            out.append(RESIDUAL * D * n if case["gate"] == "rows" else (RESIDUAL * D * n).sum(0))
    return out
