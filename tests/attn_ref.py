"""Plain 64-bit references of the attention block (numpy, on the host) and the error bounds of its kernels, used by the
GPU tests.  Nothing here calls the library."""
import math

import numpy as np

# unit roundoff of the 16-bit types (half a unit in the last place, relative) and half their smallest step
ROUND = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def rotate(x, pos, table, interleaved, inverse=False):
    """x [tokens][heads][D], in x's own precision (fp64, or fp32 with every product and sum rounded by itself)."""
    half = table.shape[2]
    t = table.astype(x.dtype)[pos]
    c, s = t[:, None, 0], t[:, None, 1] * (-1 if inverse else 1)
    y = x.copy()
    ia, ib = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), half + np.arange(half))
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def table64(positions, rot, theta=1e4, factor=1.0, low=1.0, high=4.0, original=0.0, magnitude=1.0):
    f = theta ** (-2.0 * np.arange(rot // 2) / rot)
    g = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1) if original else np.zeros_like(f)
    f = (1 - g) * f / factor + g * f
    angle = np.arange(positions)[:, None] * f
    return magnitude * np.stack([np.cos(angle), np.sin(angle)], 1)


def bf16(x):
    """fp32 rounded to bf16, as fp32."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x).astype(np.float32)


def quantise(x, kind):
    """Codes and scales of x [..][D], fp32, by the format's definition in fp32 arithmetic: codes as int8, scales [..]
    (i8) or [..][2] (i4)."""
    x = x.astype(np.float32)
    top = np.float32(127 if kind == "i8" else 7)
    parts = x.reshape(*x.shape[:-1], 1 if kind == "i8" else 2, -1)
    with np.errstate(all="ignore"):
        a = np.max(np.abs(parts), axis=-1)
        a = np.where(np.isnan(parts).any(-1), np.float32(np.nan), a)
        scale = a / top
        if kind == "i4":
            scale = bf16(scale)
        scale = np.where(a < np.float32(1e-30), np.float32(0), scale)
        inv = np.where(scale > 0, np.float32(1) / scale, np.float32(0))
        code = np.clip(np.rint(parts * inv[..., None]), -top, top)
    fine = np.isfinite(a)
    scale = np.where(fine, scale, np.float32(np.nan))
    code = np.where(fine[..., None], code, 0).reshape(x.shape).astype(np.int8)
    return code, scale[..., 0] if kind == "i8" else scale


def dequantise(code, scale, kind):
    """Values in fp32, every product rounded."""
    if kind == "i8":
        return code.astype(np.float32) * scale[..., None]
    parts = code.astype(np.float32).reshape(*code.shape[:-1], 2, -1)
    return (parts * scale[..., None]).reshape(code.shape)


def attention(q, k, v, last, scale):
    """fp64: q [n][Hq][D], k and v [m][H][D]; row i sees keys j <= last[i] (and j with a finite place: `k` holds only
    those).  Returns out, lse, sum p |v| / sum p, and the largest scale * sum |q||k| of each row."""
    n, hq, d = q.shape
    m, h = k.shape[:2]
    out, mag = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, top = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for x in range(hq):
        kk, vv = k[:, x * h // hq], v[:, x * h // hq]
        s = scale * (q[:, x] @ kk.T)
        seen = np.arange(m)[None] <= np.asarray(last)[:, None]
        any_ = seen.any(1)
        if not any_.any():
            continue
        s = np.where(seen, s, -np.inf)
        mx = np.where(any_, np.max(s, axis=1, initial=-np.inf), 0)
        p = np.exp(s - mx[:, None])
        l = p.sum(1)
        w = np.divide(p, l[:, None], out=np.zeros_like(p), where=l[:, None] > 0)
        out[:, x], mag[:, x] = w @ vv, w @ np.abs(vv)
        lse[any_, x] = (mx + np.log(np.where(l > 0, l, 1)))[any_]
        top[:, x] = np.max(np.where(seen, scale * (np.abs(q[:, x]) @ np.abs(kk).T), 0), axis=1, initial=0)
    return out, lse, mag, top


def bounds(out, lse, mag, top, keys, d, weights, dtype, vmax):
    """Largest errors of out and lse.  Scores: fp32 sums of d products and a few roundings, so off by at most
    delta = top (d + 8) 2^-24 + 2^-21; a weight by that, its own rounding to `weights` and the exponential's; the fp32
    sums over the keys by keys 2^-24; the result is rounded once.  A weight below the 16-bit type's smallest normal is
    off by half its smallest step against a largest weight of at least 1."""
    delta = top * (d + 8) * 2.0 ** -24 + 2.0 ** -21
    u = ROUND[weights] + keys * 2.0 ** -23 + 2.0 ** -20
    o = mag * (u + 2 * delta[..., None]) + ROUND[dtype] * np.abs(out) + keys * TINY[weights] * 4 * vmax + TINY[dtype]
    z = delta + keys * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))
    return o, z


def check(got_out, got_lse, ref, keys, weights, dtype, vmax):
    out, lse, mag, top = ref
    o, z = bounds(out, lse, mag, top, keys, out.shape[-1], weights, dtype, vmax)
    err = np.abs(got_out - out)
    assert not np.isnan(got_out).any()
    assert (err <= o).all(), f"out off by {np.max(err / o):.3g} times its bound"
    if got_lse is not None:
        assert np.array_equal(np.isneginf(got_lse), np.isneginf(lse))
        fine = np.isfinite(lse)
        e = np.abs(got_lse[fine] - lse[fine]) / z[fine]
        assert np.isfinite(got_lse[fine]).all() and (e <= 1).all(), f"lse off by {e.max():.3g} times its bound"
    return float(np.max(err / o)) if err.size else 0.0
