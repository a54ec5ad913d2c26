"""The float64 statements that the row calls are compared with, put together as a training step, against differences of the step's loss:
norm -> layer with adapters -> norm of its output, gate, residual -> norm; the loss is linear in the last residual stream and the last x."""
import numpy as np

import rows_plain as plain

EPS, S, SCALE = 1e-3, 2.0, 0.7
LENGTHS, SEG, RANKS = [3, 2, 2], [0, 1, -1], [2, 3]
OFFSETS = np.concatenate([[0], np.cumsum(LENGTHS)])


def _layer(x, W0, A, B):
    y = x @ W0.T
    for g, e in enumerate(SEG):
        if e >= 0:
            r = slice(OFFSETS[g], OFFSETS[g + 1])
            y[r] += S * (x[r] @ A[e].T) @ B[e].T
    return y


def _step(p):
    x = plain.norm_x(p["h0"], p["w1"], EPS)
    o = _layer(x, p["W0"], [p["A0"], p["A1"]], [p["B0"], p["B1"]])
    h1, _ = plain.norm_h(p["h0"], o, p["w2"], p["gate"], SCALE, EPS)
    return x, o, h1, plain.norm_x(h1, p["w3"], EPS)


def test_gradients_of_a_step_are_differences():
    rng = np.random.default_rng(7)
    T, d = sum(LENGTHS), 12
    p = {"h0": rng.standard_normal((T, d)), "W0": 0.3 * rng.standard_normal((d, d)), "gate": rng.standard_normal(d)}
    for e, r in enumerate(RANKS):
        p[f"A{e}"], p[f"B{e}"] = 0.3 * rng.standard_normal((r, d)), 0.3 * rng.standard_normal((d, r))
    for k in (1, 2, 3):
        p[f"w{k}"] = 1 + 0.1 * rng.standard_normal(d)
    g_h, g_x = rng.standard_normal((T, d)), rng.standard_normal((T, d))

    def loss(q):
        _, _, h1, x2 = _step(q)
        return (h1 * g_h).sum() + (x2 * g_x).sum()

    x, o, h1, _ = _step(p)
    back = plain.norm_backward(h1, o, p["w2"], p["w3"], p["gate"], SCALE, EPS, g_x, g_h)
    ents = [(r, S, p[f"A{e}"], p[f"B{e}"]) for e, r in enumerate(RANKS)]
    (dA0, dB0, _, _), (dA1, dB1, _, _) = plain.gradients(x, back["do"], ents, OFFSETS, SEG)
    dx = _layer(back["do"], p["W0"].T, [p["B0"].T, p["B1"].T], [p["A0"].T, p["A1"].T])
    first = plain.norm_backward(p["h0"], None, None, p["w1"], None, 1.0, EPS, dx, back["dh"])
    want = {"h0": first["dh"], "A0": dA0, "A1": dA1, "B0": dB0, "B1": dB1, "w1": first["dw_pre"], "w2": back["dw_post"], "w3": back["dw_pre"], "gate": back["dgate"]}
    for name, ref in want.items():
        for k in np.ndindex(ref.shape):
            two = []
            for move in (1e-6, -1e-6):
                q = dict(p)
                q[name] = p[name].copy()
                q[name][k] += move
                two.append(loss(q))
            # (a difference of two losses of a few hundred, good to 2^-52 of it each, over 2e-6: 1e-7)
            assert abs((two[0] - two[1]) / 2e-6 - ref[k]) < 1e-6 * max(1.0, abs(ref[k])), (name, k)
