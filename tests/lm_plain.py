"""The operators of the 8-bit layer step of a language model, from their definitions, in numpy float64 (test infrastructure)."""
import numpy as np
import torch

TOP = {"e4m3": (1.75, 8, -6, 3), "e5m2": (1.75, 15, -14, 2)}   # largest = 1.75 * 2^8 or 2^15, smallest normal exponent, mantissa bits
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative


def draws(n, seed):
    """16 bits of the counter-based generator for each of the flat positions 0 .. n-1."""
    def mix(x):
        x = x ^ (x >> np.uint32(16))
        x = x * np.uint32(0x6A09E667)
        x = x ^ (x >> np.uint32(15))
        x = x * np.uint32(0xBB67AE85)
        return x ^ (x >> np.uint32(16))

    seed &= 2 ** 64 - 1
    i = np.arange(n, dtype=np.uint64)
    with np.errstate(over="ignore"):
        phi = np.uint32(0x9E3779B9)
        h = mix((i >> np.uint64(2)).astype(np.uint32) * phi + np.uint32(seed & 0xFFFFFFFF)) ^ np.uint32(seed >> 32)
        w = mix(h + phi * (1 + ((i >> np.uint64(1)) & np.uint64(1)).astype(np.uint32)))
    return np.where(i & np.uint64(1), w >> np.uint32(16), w & np.uint32(0xFFFF)).astype(np.int64)


def quantize(x, fmt, rows=1, r=None):
    """(codes as values, scale bytes) of a float64 matrix with blocks of rows x 128; r: 16 random bits an entry, or None."""
    top, emax, emin, man = TOP[fmt]
    R, C = x.shape
    nr, nc = -(-R // rows), -(-C // 128)
    full = np.zeros((nr * rows, nc * 128))
    full[:R, :C] = x
    finite = np.where(np.isfinite(full), np.abs(full), 0.0)
    amax = finite.reshape(nr, rows, nc, 128).max(axis=(1, 3))
    m, e = np.frexp(amax)                      # amax = m 2^e, 0.5 <= m < 1
    E = np.clip(e - 1 - emax + (2 * m > top), -127, 127)
    E = np.where(amax == 0, 0, E)
    wide = np.repeat(np.repeat(E, rows, axis=0), 128, axis=1)
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.ldexp(full, -wide)
        ulp = np.ldexp(1.0, np.maximum(np.frexp(np.where(np.isfinite(t), t, 0.0))[1] - 1, emin) - man)
        u = np.abs(t) / ulp
        if r is None:
            k = np.rint(u)                     # nearest even
        else:
            rr = np.zeros(full.shape)
            rr[:R, :C] = r.reshape(R, C)
            k = np.floor(u) + ((u - np.floor(u)) * 65536 > rr + 0.5)
        q = np.copysign(k * ulp, t)
    q = np.where(np.isfinite(full), q, np.nan if fmt == "e4m3" else full)
    s = np.full((nr * rows, -(-nc // 4) * 4), 127, np.uint8)
    s[:, :nc] = np.repeat(E + 127, rows, axis=0)
    return q[:R], s[:R]


def values(q, s):
    """What codes (as values) and scale bytes stand for, [R, 128 * blocks]."""
    nc = q.shape[1] // 128
    return q * np.repeat(np.exp2(s[:, :nc].astype(np.float64) - 127), 128, axis=1)


def kept(n, p, seed):
    """keep / (1 - p) of each flat position, p in steps of 2^-16."""
    cut = int(np.rint(p * 65536))
    return (draws(n, seed) >= cut) * (65536.0 / (65536 - cut) if cut < 65536 else 0.0)


def dropout(x, p, seed, residual=None):
    k = kept(x.size, p, seed).reshape(x.shape)
    y = np.where(k > 0, x * k, 0.0)
    return y if residual is None else residual + y


def norm_fwd(res, h, w_post, gate, w_pre, eps, rs, bs, keep):
    """(res_out, y, 1/rms of h, 1/rms of res_out); keep: factors of every position, or 1."""
    T = res.shape[0]
    r, s1 = res, np.ones(T)
    if h is not None:
        u = h
        if w_post is not None:
            s1 = 1 / np.sqrt((h * h).mean(axis=1) + eps)
            u = h * s1[:, None] * w_post
        if gate is not None:
            u = u * np.repeat(gate, T // gate.shape[0], axis=0)
        r = rs * res + bs * np.where(keep != 0, u * keep, 0.0)
    s2 = 1 / np.sqrt((r * r).mean(axis=1) + eps)
    return r, (None if w_pre is None else r * s2[:, None] * w_pre), s1, s2


def norm_bwd(dy, dres_out, r, h, s1, s2, w_post, gate, w_pre, rs, bs, keep, size=False):
    """Gradients (dres, dh, dgate, dw_post, dw_pre).  size: the same sums over absolute values instead, the measure of a rounding error."""
    f = np.abs if size else (lambda v: v)
    minus = (lambda a, b: a + b) if size else (lambda a, b: a - b)
    T, D = r.shape
    dr, dw_pre = np.zeros((T, D)), None
    if dres_out is not None:
        dr = dr + f(dres_out)
    if w_pre is not None:
        n, dn = f(r * s2[:, None]), f(dy * w_pre)
        dr = dr + s2[:, None] * minus(dn, n * (dn * n).mean(axis=1, keepdims=True))
        dw_pre = (f(dy) * n).sum(axis=0)
    if h is None:
        return dr * f(rs), None, None, None, dw_pre
    dv = dr * f(bs) * keep
    m = f(h * s1[:, None])
    wp = f(w_post) if w_post is not None else 1.0
    dgate, dw_post, du = None, None, dv
    if gate is not None:
        G = gate.shape[0]
        dgate = (dv * m * wp).reshape(G, T // G, D).sum(axis=1)
        du = dv * np.repeat(f(gate), T // G, axis=0)
    dh = du
    if w_post is not None:
        dw_post = (du * m).sum(axis=0)
        dm = du * wp
        dh = s1[:, None] * minus(dm, m * (dm * m).mean(axis=1, keepdims=True))
    return dr * f(rs), dh, dgate, dw_post, dw_pre


def host(t):
    return None if t is None else t.to(torch.float32).cpu().numpy().astype(np.float64)


def within(got, want, off, what):
    """got (tensor) within `off` of `want` everywhere."""
    assert tuple(got.shape) == tuple(want.shape), what
    bad = ~(np.abs(host(got) - want) <= off)
    if bad.any():
        at = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off; at %s %r, expected %r within %r" % (what, bad.sum(), bad.size, at, host(got)[at], want[at],
                                                                                   np.broadcast_to(off, want.shape)[at]))
