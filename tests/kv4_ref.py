"""The 4-bit cache and its attention in float64 numpy, from the definition in
include/spec_ops.h, and the byte order of csrc/kv4_layout.h (not collected: no
test_ prefix)."""

import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
SIGNED = np.concatenate([LEVELS, -LEVELS])


def block_bytes(hd):
    return 8 * hd + hd // 2


def k_place(t, d, hd):
    """(byte, nibble, scale byte) of dim d of token t's key in its block."""
    s, g, i = d // 32, d // 8 % 4, d % 8
    h, j = t // 4 % 2, t % 4 + 4 * (t // 8)
    unit = ((h * 4 + g) * 8 + j) * 16 if hd == 128 else ((g * 8 + j) * 2 + h) * 8
    return unit + 4 * s + i // 2, i % 2, 8 * hd + (j * 2 + h) * (hd // 32) + s


def v_place(t, d, hd):
    b, i = d // 32, d % 16
    return ((b // 2 * 2 + t // 8) * 16 + i) * 16 + 8 * (b % 2) + t % 8, d % 32 // 16, 8 * hd + (t // 8 * (hd // 32) + b) * 8 + t % 8


def quantise(x):
    """(codes, scale bytes per block of 32) of fp64 x [..., hd]."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    e = np.full(top.shape, -126)
    for i in np.ndindex(*top.shape):
        if bad[i]:
            continue
        while 6.0 * 2.0 ** e[i] < top[i]:
            e[i] += 1
    r = np.abs(np.where(bad[..., None], 0, b)) * 2.0 ** -e[..., None].astype(np.float64)
    dist = np.abs(r[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = np.where(np.signbit(b), code + 8, code)
    return code.reshape(x.shape), np.where(bad, 255, e + 127)


def values(codes, scales):
    v = SIGNED[codes] * 2.0 ** (np.repeat(scales, 32, -1).astype(np.float64) - 127)
    return np.where(np.repeat(scales, 32, -1) == 255, np.nan, v)


def held(x):
    return values(*quantise(x))


def put(pages, slot, x, place):
    """Write fp64 vectors x [R, Hkv, hd] into the slots of uint8 pages [P, Hkv, block bytes]."""
    hd = x.shape[-1]
    codes, scales = quantise(x)
    for r, sl in enumerate(slot):
        t = sl % 16
        for d in range(hd):
            byte, nib, sb = place(t, d, hd)
            blk = pages[sl // 16]
            blk[:, byte] = (blk[:, byte] & (0xF0 if nib == 0 else 0x0F)) | (codes[r, :, d] << (4 * nib))
            blk[:, sb] = scales[r, :, d // 32]


def get(pages, slot, hd, place):
    """fp64 [n, Hkv, hd] held in the slots."""
    slot = np.asarray(slot)
    out = np.empty((len(slot), pages.shape[1], hd))
    with np.errstate(invalid="ignore"):
        for t in range(16):
            rows = np.nonzero(slot % 16 == t)[0]
            if not len(rows):
                continue
            blocks = pages[slot[rows] // 16]
            for d in range(hd):
                byte, nib, sb = place(t, d, hd)
                s = blocks[:, :, sb]
                v = SIGNED[(blocks[:, :, byte] >> (4 * nib)) & 15] * 2.0 ** (s.astype(np.float64) - 127)
                out[rows, :, d] = np.where(s == 255, np.nan, v)
    return out


def rotate(x, pos, theta):
    """fp64 rotary embedding of [R, H, hd]."""
    half = x.shape[-1] // 2
    a = np.asarray(pos, np.float64)[:, None] * float(np.float32(theta)) ** (-np.arange(half) / half)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def attention(q, k, v, pos0):
    """One sequence: q [r, Hq, hd], k, v [n, Hkv, hd] fp64, causal from position pos0.  Returns the
    output [r, Hq, hd], sum p |v| and the largest sum |q k| / sqrt(hd) of any score (for error bounds)."""
    r, hq, hd = q.shape
    G = hq // k.shape[1]
    out, mag, big = np.empty(q.shape), np.empty(q.shape), 0.0
    hidden = np.arange(len(k))[None] > pos0 + np.arange(r)[:, None]
    for h in range(hq):
        kk, vv = k[:, h // G], v[:, h // G]
        s = np.where(hidden, -np.inf, q[:, h] @ kk.T / np.sqrt(hd))
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h], mag[:, h] = p @ vv, p @ np.abs(vv)
        big = max(big, float(np.where(hidden, 0, np.abs(q[:, h]) @ np.abs(kk).T).max()) / np.sqrt(hd))
    return out, mag, big


def attention_rows(q, k, v, pos0):
    """As attention(), of the keys that a row sees alone (what later keys hold does not enter), with the
    largest sum |q k| / sqrt(hd) of each row and head [r, Hq, 1]."""
    r, hq, hd = q.shape
    G = hq // k.shape[1]
    out, mag, big = np.empty(q.shape), np.empty(q.shape), np.empty((r, hq, 1))
    with np.errstate(invalid="ignore", over="ignore"):
        for g in range(k.shape[1]):
            kt, vv = np.ascontiguousarray(k[:, g].T), np.ascontiguousarray(v[:, g])
            ka, va = np.abs(kt), np.abs(vv)
            for i in range(r):
                n = pos0 + i + 1
                rows = q[i, g * G:(g + 1) * G]
                s = rows @ kt[:, :n] / np.sqrt(hd)
                p = np.exp(s - s.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[i, g * G:(g + 1) * G], mag[i, g * G:(g + 1) * G] = p @ vv[:n], p @ va[:n]
                big[i, g * G:(g + 1) * G, 0] = (np.abs(rows) @ ka[:, :n]).max(1) / np.sqrt(hd)
    return out, mag, big
