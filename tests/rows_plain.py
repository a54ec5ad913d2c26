"""Plain float64 / integer statements of the row operators (checkpoints, block norms, gradients from rows), for the tests."""
import numpy as np

FORMS = ("int8", "e4m3")


def widen(bits):
    """bf16 bits (uint16) -> float64."""
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16(x):
    """float64 -> bf16 bits, nearest even (finite values within range)."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) & 0xFFFF).astype(np.uint16)


def e4m3_values():
    """The 256 values of FP8 E4M3 (no infinities; S.1111.111 is NaN)."""
    v = np.empty(256)
    for b in range(256):
        s, e, m = -1.0 if b & 128 else 1.0, (b >> 3) & 15, b & 7
        v[b] = s * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        if e == 15 and m == 7:
            v[b] = np.nan
    return v


def encode(bits, form):
    """-> (data uint8 [T][pitch], scales uint8 [groups][T][4])."""
    T, d = bits.shape
    nb = (d + 31) // 32
    v = np.zeros((T, nb * 32))
    v[:, :d] = widen(bits)
    v = v.reshape(T, nb, 32)
    scale = np.zeros((T, nb), np.int64)
    q = np.zeros((T, nb, 32), np.uint8)
    table = e4m3_values()[:127]                                       # the positive finite ones, ascending
    least = 0 if form == "int8" else 3
    for t in range(T):
        for k in range(nb):
            blk = v[t, k]
            if not np.isfinite(blk).all():
                scale[t, k] = 255
                continue
            amax = np.abs(blk).max()
            if amax == 0:
                b = 0
            else:
                e = np.frexp(amax)[1] - 1                              # binade
                b = e - 6 + 127 if form == "int8" else e - 8 + 127 + (1 if amax > 448 * 2.0 ** (e - 8) else 0)
            b = max(b, least)
            scale[t, k] = b
            s = blk * 2.0 ** (127 - b)
            if form == "int8":
                q[t, k] = np.clip(np.rint(s), -127, 127).astype(np.int8).view(np.uint8)
            else:
                a = np.minimum(np.abs(s), 240.0 if b == 247 else 448.0)   # (256 units of 2^120 would be 2^128: not in bf16)
                hi = np.clip(np.searchsorted(table, a), 1, 126)        # nearest, ties to the even code
                lo = hi - 1
                up = (a - table[lo] > table[hi] - a) | ((a - table[lo] == table[hi] - a) & (hi % 2 == 0))
                q[t, k] = np.where(up, hi, lo).astype(np.uint8) | (np.signbit(s).astype(np.uint8) << 7)
    groups = (d + 127) // 128
    out = np.zeros((T, groups * 4), np.uint8)
    out[:, :nb] = scale
    return q.reshape(T, nb * 32), np.ascontiguousarray(out.reshape(T, groups, 4).transpose(1, 0, 2))


def decode(data, scales, d, form):
    """-> float64 [T][d]."""
    T, pitch = data.shape
    b = scales.transpose(1, 0, 2).reshape(T, -1)[:, :pitch // 32].astype(np.int64)
    q = data.view(np.int8).astype(np.float64) if form == "int8" else e4m3_values()[data]
    s = np.where(b == 255, np.nan, 2.0 ** (b - 127.0))
    return (q.reshape(T, -1, 32) * s[..., None]).reshape(T, pitch)[:, :d]


def kept(bits, form):
    """What a checkpoint of these rows stands for; bf16 rows stand for themselves."""
    return widen(bits) if form == "bf16" else decode(*encode(bits, form), bits.shape[1], form)


def norm_h(h, o, w_post, gate, scale, eps):
    """h' before its rounding, and the size of what was added up."""
    n = o
    if w_post is not None:
        n = o / np.sqrt((o * o).mean(1, keepdims=True) + eps) * w_post
    add = scale * (n if gate is None else gate * n)
    return h + add, np.abs(h) + np.abs(add)


def norm_x(h, w_pre, eps):
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * w_pre


def norm_backward(h, o, w_post, w_pre, gate, scale, eps, dx, dh_new):
    """Gradients at h' = h, and beside each the sum of the absolute values of what it is added up from."""
    r = {}
    D, mD = (np.zeros_like(h) if dh_new is None else dh_new), 0.0
    mD = np.abs(D)
    if dx is not None:
        rho = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
        hh, g = h * rho, dx * w_pre
        D = D + rho * (g - hh * (g * hh).mean(1, keepdims=True))
        mD = mD + rho * (np.abs(g) + np.abs(hh) * np.abs(g * hh).mean(1, keepdims=True))
        r["dw_pre"], r["m_dw_pre"] = (dx * hh).sum(0), np.abs(dx * hh).sum(0)
    r["dh"], r["m_dh"] = D, mD
    if o is not None:
        ro = 1.0 if w_post is None else 1 / np.sqrt((o * o).mean(1, keepdims=True) + eps)
        oo, w = o * ro, 1.0 if w_post is None else w_post
        gt = 1.0 if gate is None else gate
        dn, mdn = scale * gt * D, abs(scale) * np.abs(gt) * mD
        r["dgate_rows"], r["m_dgate_rows"] = scale * D * oo * w, abs(scale) * mD * np.abs(oo * w)
        r["dgate"], r["m_dgate"] = r["dgate_rows"].sum(0), r["m_dgate_rows"].sum(0)
        r["dw_post"], r["m_dw_post"] = (dn * oo).sum(0), (mdn * np.abs(oo)).sum(0)
        go, mgo = dn * w, mdn * np.abs(w)
        if w_post is None:
            r["do"], r["m_do"] = go, mgo
        else:
            r["do"] = ro * (go - oo * (go * oo).mean(1, keepdims=True))
            r["m_do"] = ro * (mgo + np.abs(oo) * (mgo * np.abs(oo)).mean(1, keepdims=True))
    return r


def gradients(x, dy, entries, offsets, seg_entry):
    """Per entry (rank, scale, A float64, B float64): (dA, dB) and the sums of the absolute values of their terms."""
    out = []
    for e, (r, s, A, B) in enumerate(entries):
        dA, dB, mA, mB = (np.zeros(z.shape) for z in (A, B, A, B))
        for g, k in enumerate(seg_entry):
            if k == e:
                xs, ds = x[offsets[g]:offsets[g + 1]], dy[offsets[g]:offsets[g + 1]]
                dA += s * (ds @ B).T @ xs
                dB += s * ds.T @ (xs @ A.T)
                mA += abs(s) * (np.abs(ds) @ np.abs(B)).T @ np.abs(xs)
                mB += abs(s) * np.abs(ds).T @ (np.abs(xs) @ np.abs(A).T)
        out.append((dA, dB, mA, mB))
    return out
