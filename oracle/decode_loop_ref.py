"""Plain CPU statements of the decode loop's operators: rotary positions, page assignment, the 4-bit format and its page
layout, attention over it.  float64 and Python integers, written from the definitions; test infrastructure only."""
import math

import numpy as np

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- rotary -----------------------------------------------------------------------------------
def frequencies(R, theta=10000.0, scaling="none", factor=1.0, original_tokens=0, beta_fast=32.0, beta_slow=1.0):
    """(radians per position of each pair, magnitude)"""
    if scaling == "base" and R > 2:
        theta = theta * factor ** (R / (R - 2))
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        out = []
        for x in f:
            turns = original_tokens * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)))
            out.append(x * keep + x / factor * (1 - keep))
        return out, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def rotary(x, positions, f, R, interleaved=False, magnitude=1.0, sections=None, inverse=False):
    """x float64 [B, T, H, d], positions int [streams, B, T]; returns (y, |x0| + |x1| of each element's pair, angles)."""
    x = np.asarray(x, np.float64)
    f = np.asarray(f, np.float64)
    sections = [R // 2] if sections is None else list(sections)
    stream = np.repeat(np.arange(len(sections)), sections)
    angle = np.asarray(positions, np.float64)[stream].transpose(1, 2, 0) * f            # [B, T, R/2]
    c, s = np.cos(angle)[:, :, None] * magnitude, np.sin(angle)[:, :, None] * magnitude
    if inverse:
        s = -s
    i0 = np.arange(0, R, 2) if interleaved else np.arange(R // 2)
    i1 = i0 + 1 if interleaved else i0 + R // 2
    y, size = x.copy(), np.abs(x)
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
    size[..., i0] = size[..., i1] = np.abs(a) + np.abs(b)
    return y, size, angle


# ---- pages ------------------------------------------------------------------------------------
def assign_pages(rows, add, table, page_size, cursor, free, slots_per_seq):
    """rows, add [B, L]; table [B, L, H, max_pages] (a changed copy is returned); free: list of pages."""
    B, L, H, most = table.shape
    table, slots = table.copy(), np.full((B, slots_per_seq), -1, np.int64)
    out = np.zeros((B, L), np.int32)
    for b in range(B):
        at = 0
        for l in range(L):
            r, a = max(0, int(rows[b, l])), max(0, int(add[b, l]))
            out[b, l] = min(r + a, (1 << 25) - 1)
            for h in range(H):
                for row in range(r, r + a):
                    p = row // page_size
                    page = -1
                    if p < most:
                        if row % page_size == 0:
                            table[b, l, h, p] = free[cursor] if 0 <= cursor < len(free) else -1
                            cursor += 1
                        page = int(table[b, l, h, p])
                    if at < slots_per_seq:
                        slots[b, at] = page * page_size + row % page_size if page >= 0 else -1
                    at += 1
    return table, slots, out, cursor


# ---- the 4-bit format -------------------------------------------------------------------------
def encode(x):
    """Codes uint8 [..., d] and scales uint8 [..., d/32] of float32 values."""
    x = np.asarray(x, np.float32)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32).astype(np.float64)
    top = np.abs(y).max(-1)
    E = np.zeros(top.shape, np.int64)
    flat = E.reshape(-1)
    for i, t in enumerate(top.reshape(-1)):
        if not math.isfinite(t):
            flat[i] = 255
            continue
        e = math.frexp(t)[1] - 1 - 2 if t > 0 else -200
        if t >= math.ldexp(7.0, e):
            e += 1
        flat[i] = min(252, max(2, e + 127))
    codes = np.zeros(y.shape, np.uint8)
    fine = E < 255
    size = np.abs(np.where(fine[..., None], y, 0.0)) * np.exp2(127.0 - E)[..., None]
    distance = np.abs(size[..., None] - np.array(E2M1))
    # the nearest; of two as near the even code
    best = distance.min(-1, keepdims=True)
    for code in (7, 5, 3, 1, 6, 4, 2, 0):
        codes[distance[..., code] == best[..., 0]] = code
    codes |= np.where(fine[..., None] & np.signbit(y), 8, 0).astype(np.uint8)
    return codes.reshape(x.shape), E.astype(np.uint8)


def decode(codes, E):
    value = np.array(E2M1 + tuple(-v for v in E2M1))[codes]
    E = E.astype(np.float64)
    unit = np.where(E == 255, np.nan, np.exp2(E - 127))
    return (value.reshape(*codes.shape[:-1], codes.shape[-1] // 32, 32) * unit[..., None]).reshape(codes.shape)


def grid(x):
    return decode(*encode(x))


def _places(d, slot):
    """Byte of K codes / V codes of each pair of columns, of K scales / V scales of each block, in a flat cache."""
    base, i = slot // 16 * 17 * d, slot % 16
    pair, block = np.arange(d // 2), np.arange(d // 32)
    kc = base + i * (d // 2) + pair
    per = d // 32                                   # bytes of a row in one place: d / 16 columns
    vc = base + 8 * d + (i // 4) * 2 * d + (pair // per) * 4 * per + (i % 4) * per + pair % per
    return kc, vc, base + 16 * d + block * 16 + i, base + 16 * d + d // 2 + (i // 4) * (d // 8) + block * 4 + i % 4


def store(pages, slots, K, V):
    """pages: flat uint8, changed in place; slots [n]; K, V float32 [n, d]."""
    d = K.shape[-1]
    for slot, k, v in zip(slots, K, V):
        if slot < 0 or int(slot) // 16 * 17 * d + 17 * d > pages.size:
            continue
        kc, vc, ks, vs = _places(d, int(slot))
        for rows, at, scales in ((k, kc, ks), (v, vc, vs)):
            c, E = encode(rows)
            pages[at] = c[0::2] | (c[1::2] << 4)
            pages[scales] = E
    return pages


def load(pages, slots, d):
    out = np.zeros((2, len(slots), d))
    for n, slot in enumerate(slots):
        if slot < 0 or int(slot) // 16 * 17 * d + 17 * d > pages.size:
            continue
        kc, vc, ks, vs = _places(d, int(slot))
        for which, (at, scales) in enumerate(((kc, ks), (vc, vs))):
            c = np.stack((pages[at] & 15, pages[at] >> 4), -1).reshape(-1)
            out[which, n] = decode(c, pages[scales])
    return out[0], out[1]


# ---- attention --------------------------------------------------------------------------------
def attend(q, K, V, scale):
    """q [G, d], K, V [n, d] float64: (out [G, d], sum p |v| [G, d], largest sum |q k| and |logit| [G])."""
    if K.shape[0] == 0:
        z = np.zeros_like(q)
        return z, z, np.zeros(len(q)), np.zeros(len(q))
    logit = q @ K.T * scale
    p = np.exp(logit - logit.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return p @ V, p @ np.abs(V), (np.abs(q) @ np.abs(K.T)).max(1) * abs(scale), np.abs(logit).max(1)
