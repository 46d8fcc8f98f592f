"""fp64 restatement of rotary positions, the paged key/value cache and attention over it.

The cache's bytes are taken apart by their documented layout, one key at a time.
"""
import math

import numpy as np

from . import fp8pv, mxfp4


def rotary(x, positions, inv_freq, interleaved=False, magnitude=1.0, inverse=False):
    """x [..., H, N, d] (positions [..., N]): the first 2 len(inv_freq) channels turned, pair by pair."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    half = len(inv_freq)
    t = np.asarray(positions, dtype=np.float64)[..., None, :, None] * np.asarray(inv_freq, dtype=np.float64)
    c, s = np.cos(t), np.sin(t) * (-1.0 if inverse else 1.0)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = magnitude * (x[..., a] * c - x[..., b] * s)
    y[..., b] = magnitude * (x[..., a] * s + x[..., b] * c)
    return y


def block_quantize(x, fp8):
    """Code bytes and scale bytes of x [..., d], 32 values along d per block."""
    return fp8pv.quantize(x) if fp8 else mxfp4.quantize(x)


def values(codes, scales, fp8):
    """What code bytes [..., b] under scales [..., d / 32] stand for; NaN under byte 255."""
    if not fp8:
        return mxfp4.dequantize(codes, scales)
    return np.where(np.repeat(np.asarray(scales) == 255, 32, axis=-1), np.nan, fp8pv.dequantize(codes, scales))


def key_rows(cache, slot):
    """(k_codes, k_scales, v_codes, v_scales) rows [H, ...] of one slot, in the order of d."""
    k_codes, k_scales, v_codes, v_scales = cache
    page, off = divmod(int(slot), k_codes.shape[2])
    H = k_codes.shape[1]
    v = v_codes[page, :, off // 8, :, off % 8].reshape(H, -1)
    return k_codes[page, :, off], k_scales[page, :, off], v, v_scales[page, :, off // 8, :, off % 8]


def key_values(cache, slots, fp8):
    """K and V [m, H, d] of slots."""
    rows = [key_rows(cache, s) for s in slots]
    kc, ks, vc, vs = (np.stack(r) for r in zip(*rows))
    return values(kc, ks, fp8), values(vc, vs, fp8)


def attention(q, k, v, visible, softmax_scale):
    """q [T, Hq, d], k and v [n, H, d], visible [T, n].  Returns O [T, Hq, d], the log
    normaliser [T, Hq], and what error bounds need: the weighted mean of |v - O| and of |v|
    [T, Hq, d], and the largest sum of |q| |k| of a score [T, Hq].  Keys that a row does not see are left out of it."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1] if len(k) else 1
    out, lse = np.zeros((T, Hq, d)), np.full((T, Hq), -math.inf)
    spread, size, reach = np.zeros((T, Hq, d)), np.zeros((T, Hq, d)), np.zeros((T, Hq))
    for t in range(T):
        seen = np.flatnonzero(visible[t])
        if len(seen) == 0:
            continue
        for h in range(Hq):
            kk, vv = k[seen, h // G], v[seen, h // G]
            z = kk @ q[t, h] * softmax_scale
            top = z.max()
            w = np.exp(z - top)
            lse[t, h] = top + math.log(w.sum())
            w = w / w.sum()
            out[t, h] = w @ vv
            spread[t, h] = w @ np.abs(vv - out[t, h])
            size[t, h] = w @ np.abs(vv)
            reach[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * softmax_scale
    return out, lse, spread, size, reach


def causal_mask(T, n, length):
    """Token t of T stands at position length - T + t."""
    return np.arange(n)[None, :] <= (length - T + np.arange(T))[:, None]


def tree_mask(words, T, n, length):
    """words [T, W] of 64 bits: the keys before the new tokens, and the new ones of set bits."""
    u = np.arange(n) - (length - T)
    see = np.broadcast_to(u < 0, (T, n)).copy()
    for t in range(T):
        for j in np.flatnonzero((u >= 0) & (u < 64 * words.shape[1])):
            see[t, j] = bool(int(words[t, u[j] // 64]) >> int(u[j] % 64) & 1)
    return see


def assign(table, held, lengths, ring, counts, page, tokens, new=None, shared=None):
    """One step's pages, slots and positions, sequence by sequence.  table (a list of rows) and ring (a list) are
    changed; returns slots, positions, starts, lengths and counts after the step."""
    B, width = len(table), len(table[0])
    capacity, (taken, returned) = width * page, counts
    new = [tokens // B] * B if new is None else [max(0, n) for n in new]
    shared = [0] * B if shared is None else [min(max(s, 0), capacity) // page for s in shared]
    room = min(max(returned - taken, 0), len(ring))
    slots, positions, starts, after, gone = [], [], [0], [], []
    asked = 0
    for b in range(B):
        keys, want = min(max(held[b], 0), capacity), max(lengths[b], 0)
        had, now = max(-(-keys // page), shared[b]), max(-(-want // page), shared[b])
        served = want <= capacity
        if served and now > had:
            asked += now - had
            served = asked <= room
            for j in range(had, now if served else had):
                table[b][j] = ring[taken % len(ring)]
                taken += 1
        elif served:
            gone += table[b][now:had]
        for t in range(min(new[b], tokens - len(slots))):
            at = lengths[b] - new[b] + t
            ok = served and shared[b] * page <= at < capacity
            number = table[b][at // page] if ok else -1
            slots.append(number * page + at % page if number >= 0 else -1)
            positions.append(max(at, 0))
        starts.append(len(slots))
        after.append(want if served else keys)
    for j, p in enumerate(gone):
        ring[(returned + j) % len(ring)] = p
    rest = tokens - len(slots)
    return slots + [-1] * rest, positions + [0] * rest, starts, after, [taken, returned + len(gone)]


def shaped_mask(T, n, length, window=0, prefix=0):
    """Token t of T at position p = length - T + t sees keys j <= p and j < prefix, with a window only j > p - window."""
    key, at = np.arange(n)[None, :], (length - T + np.arange(T))[:, None]
    see = (key <= at) | (key < prefix)
    return see & (key > at - window) if window else see


def shaped_attention(q, k, v, visible, softmax_scale, softcap=0.0, slopes=None, length=0):
    """`attention` with z capped, softcap tanh(z / softcap), and then slopes[h] times its distance less for every key;
    the tokens stand at positions length - T ...  The sizes that error bounds need follow: as there, and the largest
    |capped score| and the largest |bias| of a row [T, Hq]."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1] if len(k) else 1
    out, lse = np.zeros((T, Hq, d)), np.full((T, Hq), -math.inf)
    spread, size = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    reach, high, bias = (np.zeros((T, Hq)) for _ in range(3))
    for t in range(T):
        seen = np.flatnonzero(visible[t])
        if len(seen) == 0:
            continue
        far = np.abs(length - T + t - seen)
        for h in range(Hq):
            kk, vv = k[seen, h // G], v[seen, h // G]
            z = kk @ q[t, h] * softmax_scale
            if softcap:
                z = softcap * np.tanh(z / softcap)
            high[t, h] = np.abs(z).max()
            if slopes is not None:
                z = z - slopes[h] * far
                bias[t, h] = np.abs(slopes[h] * far).max()
            top = z.max()
            w = np.exp(z - top)
            lse[t, h] = top + math.log(w.sum())
            w = w / w.sum()
            out[t, h] = w @ vv
            spread[t, h] = w @ np.abs(vv - out[t, h])
            size[t, h] = w @ np.abs(vv)
            reach[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * softmax_scale
    return out, lse, spread, size, reach, high, bias
