"""Oracles of the 4-bit cache and of the choice of a token, in 64 bits and plain loops.

Test infrastructure only; shares nothing with the CUDA code.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def bf16(x):
    """Nearest bf16 of each value (ties to even), as float64; through float32, which holds every bf16."""
    x = np.asarray(x, dtype=np.float32)
    bits = x.view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000
    out = bits.astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(np.isnan(x), np.nan, out)


def quantise(x, group):
    """``x`` float64 ``[..., D]`` of bf16 values.  Returns (codes int, step, lowest), the latter ``[..., D / group]``."""
    g = np.asarray(x).reshape(*x.shape[:-1], -1, group)
    codes, steps, lows = np.zeros(g.shape, dtype=np.int64), np.zeros(g.shape[:-1]), np.zeros(g.shape[:-1])
    for at in np.ndindex(*g.shape[:-1]):
        v = g[at].astype(np.float32)
        low, high = v.min() + np.float32(0), v.max()                   # one zero
        with np.errstate(all="ignore"):
            step = float(bf16((high - low) / np.float32(15)))
        if not np.all(np.isfinite(v)) or not math.isfinite(step):
            steps[at] = np.nan
            lows[at] = low
            continue
        if step < 2.0 ** -100:
            step = 0.0
        steps[at], lows[at] = step, low
        if step > 0:
            t = (v - low).astype(np.float64)                       # float32 differences; their quotients by 8-bit steps tie exactly or not at all
            codes[at] = np.minimum(15, [round(q) for q in t / step])
    return codes.reshape(x.shape), steps, lows


def place_k(t, e, d):
    """(byte of the section, high nibble) of the code of token t, element e."""
    word = (e // 8 % 4) * (d // 32) + e // 32
    return t * d // 2 + 4 * word + e % 8 // 2, e % 2


def place_v(t, e, d):
    row = t // 2 % 4 + 4 * (t % 2) + 8 * (t // 8)
    unit = e % 8
    if d == 128 and row & 2:
        unit ^= 4
    nibble = e % 32 // 8
    return row * d // 2 + unit * (d // 16) + 2 * (e // 32) + nibble // 2, nibble % 2


def slab_bytes(d, group):
    return PAGE * d + 8 * PAGE * (d // group)


def store(slab, t, k, v, group):
    """Writes token t of one KV head: ``k``, ``v`` float64 ``[D]`` of bf16 values, ``slab`` uint8."""
    d = len(k)
    for part, (x, place) in enumerate(((k, place_k), (v, place_v))):
        codes, steps, lows = quantise(x, group)
        for e in range(d):
            byte, high = place(t, e, d)
            at = part * PAGE * d // 2 + byte
            slab[at] = (slab[at] & (0x0F if high else 0xF0)) | (int(codes[e]) << (4 if high else 0))
        for j, (s, low) in enumerate(zip(steps, lows)):
            at = PAGE * d + (part * PAGE + t) * (d // group) * 4 + 4 * j
            for i, value in enumerate((s, low)):
                bits = 0x7FC0 if math.isnan(value) else int(np.float32(value).view(np.uint32)) >> 16
                slab[at + 2 * i], slab[at + 2 * i + 1] = bits & 255, bits >> 8


def _tables(d):
    return [np.array([[place(t, e, d) for e in range(d)] for t in range(PAGE)]) for place in (place_k, place_v)]


def load(slabs, d, group):
    """Keys and values of slabs uint8 ``[..., bytes]`` as ``(code, step, lowest)`` triples of arrays ``[..., 16, D]``."""
    params = np.ascontiguousarray(slabs[..., PAGE * d:]).view(np.uint16).astype(np.uint32) << 16
    params = params.view(np.float32).astype(np.float64).reshape(*slabs.shape[:-1], 2, PAGE, d // group, 2)
    out = []
    for part, table in enumerate(_tables(d)):
        byte = slabs[..., part * PAGE * d // 2 + table[..., 0]].astype(np.int64)
        code = (byte >> (4 * table[..., 1])) & 15
        step, low = (np.repeat(params[..., part, :, :, i], group, -1) for i in (0, 1))
        out.append((code, step, low))
    return out


def attend(q, k, v, scale, steer, spans):
    """One query row of one head over keys and values ``[L, D]`` that are ``(code, step, lowest)``.  Returns the output, the span masses, and
    bounds of what their rounding may come to: see ``bounds`` in the tests."""
    kc, ks, kl = k
    vc, vs, vl = v
    x = (kc * ks + kl) @ q * scale
    p = np.exp(x - x.max())
    p /= p.sum()
    out = p @ (vc * vs + vl) + steer
    size = dict(x=float((np.abs(q) * (15 * ks + np.abs(kl))).sum(1).max() * abs(scale)), coded=p @ (vc * vs), largest=float(np.abs(15 * vs + np.abs(vl)).max()),
                step=float(vs.max()), keys=len(x))
    return out, [float(p[max(0, a):max(0, b)].sum()) for a, b in spans], size


def kept(x, temperature, top_k, top_p, min_p):
    """The indices that the filters leave, and their weights; ``x`` a list of floats (NaN: -inf)."""
    x = [-math.inf if math.isnan(v) else v + 0.0 for v in x]
    top = max(x)
    order = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: (-x[i], i))
    if temperature == 0:
        return order[:1], [1.0]
    w = {i: 1.0 if x[i] == top else math.exp((x[i] - top) / temperature) for i in order}
    if 0 < top_k < len(x):
        order = order[:top_k]
    if min_p > 0:
        order = [i for i in order if w[i] >= min_p]
    if top_p < 1:
        total, before, cut = math.fsum(w[i] for i in order), 0.0, []
        for i in order:
            if cut and not before < top_p * total:
                break
            cut.append(i)
            before += w[i]
        order = cut
    order.sort()
    return order, [w[i] for i in order]


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, how far the random number is from the next border as a share of the total weight).  A token that weighs less than half of 2^-42
    has no share; of u = 0 only those decide whose weight is near that."""
    order, w = kept(x, temperature, top_k, top_p, min_p)
    if not order:
        return -1, 1.0
    total = math.fsum(w)
    if u == 0.0:
        first = next(i for i, each in enumerate(w) if each * 2.0 ** 42 >= 0.5)
        return order[first], min(abs(each * 2.0 ** 42 - 0.5) for each in w[:first + 1])
    so_far, token, gap = 0.0, None, 1.0
    for i, each in zip(order, w):
        so_far += each
        if i != order[-1] and so_far < total * (1 - 2.0 ** -40):
            gap = min(gap, abs(so_far / total - u))
        if token is None and so_far > u * total:
            token = i
    return order[-1] if token is None else token, gap
