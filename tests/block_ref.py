"""Plain 64-bit forms (numpy) of the block norms and of the microscaled 4-bit values, for
the tests; with what their float32 evaluation may be off by."""
import numpy as np

U32 = 2.0 ** -24                      # half a step of float32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def norm_fwd(res, y, gate, w_post, w_pre, scale, eps):
    """r, n, rstd_post, rstd_pre and the magnitude of r's terms."""
    p, rpo, n, rpr = y, None, None, None
    if y is None:
        r, mag = res, np.abs(res)
    else:
        if w_post is not None:
            rpo = 1.0 / np.sqrt((y * y).mean(1) + eps)
            p = y * rpo[:, None] * w_post
        if gate is not None:
            p = p * gate
        r = scale * res + p
        mag = np.abs(scale * res) + np.abs(p)
    if w_pre is not None:
        rpr = 1.0 / np.sqrt((r * r).mean(1) + eps)
        n = r * rpr[:, None] * w_pre
    return r, n, rpo, rpr, mag


def norm_bwd(dr, dn, y, r, rpo, rpr, gate, w_post, w_pre, scale):
    """dict of gradients, and of the sums of the magnitudes of each one's terms."""
    out, mag = {}, {}
    G = np.zeros_like(dn) if dr is None else dr
    mG = np.abs(G)
    if w_pre is not None:
        hat = r * rpr[:, None]
        out["dw_pre"], mag["dw_pre"] = (dn * hat).sum(0), np.abs(dn * hat).sum(0)
        wd = dn * w_pre
        G = G + rpr[:, None] * (wd - hat * (wd * hat).mean(1, keepdims=True))
        mG = mG + rpr[:, None] * (np.abs(wd) + np.abs(hat) * np.abs(wd * hat).mean(1, keepdims=True))
    out["dres"], mag["dres"] = scale * G, abs(scale) * mG
    if y is None and gate is None and w_post is None:
        out["dy"], mag["dy"] = G, mG
        return out, mag
    hat = y if w_post is None else y * rpo[:, None]
    p = hat if w_post is None else hat * w_post
    dp, mp = G, mG
    if gate is not None:
        full, mfull = G * p, mG * np.abs(p)
        if gate.ndim == 1:
            out["dgate"], mag["dgate"] = full.sum(0), mfull.sum(0)
        elif gate.shape[1] == 1:
            out["dgate"], mag["dgate"] = full.sum(1, keepdims=True), mfull.sum(1, keepdims=True)
        else:
            out["dgate"], mag["dgate"] = full, mfull
        dp, mp = G * gate, mG * np.abs(gate)
    if w_post is not None:
        out["dw_post"], mag["dw_post"] = (dp * hat).sum(0), (mp * np.abs(hat)).sum(0)
        wd, mw = dp * w_post, mp * np.abs(w_post)
        dp = rpo[:, None] * (wd - hat * (wd * hat).mean(1, keepdims=True))
        mp = rpo[:, None] * (mw + np.abs(hat) * (mw * np.abs(hat)).mean(1, keepdims=True))
    out["dy"], mag["dy"] = dp, mp
    return out, mag


# ---- microscaled 4 bits --------------------------------------------------------------------

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx_quantize(x):
    """float64 [..., K] -> (codes [..., K/2], scales [..., K/32]) uint8."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(b).all(-1)
    v = np.where(np.isfinite(b), b, 1.0)
    top = np.abs(v).max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 3, -127)
    e = np.maximum(e, -127)
    a = np.ldexp(np.abs(v), -e[..., None])
    # nearest, a tie to the even code; beyond 6 to 6
    code = np.zeros(a.shape, np.uint8)
    for i in range(7):
        mid = (E2M1[i] + E2M1[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    code |= np.signbit(v).astype(np.uint8) << 3
    code = code.reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | code[..., 1] << 4, np.where(bad, 255, e + 127).astype(np.uint8)


def mx_values(codes, scales):
    """The float64 values of codes and scales (255: NaN)."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1, 32)
    v = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v * s[..., None]).reshape(*codes.shape[:-1], -1)
