"""Plain 4-bit KV cache: the rounding, the page layout, the tables and causal attention, in numpy and 64 bits.

Shares no code with the GPU path.  Blocks of 32 dimensions hold 4-bit codes (sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6) and a power
of two that brings the block's largest magnitude into [3.5, 7) (2^-125..2^125: all values are normal in fp32); codes round to nearest, ties to the even code; a block with
a value that is not finite is NaN throughout.
"""
import math

import numpy as np

PAGE = 16
STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_block(x):
    """32 values -> (codes, biased exponent)."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return np.zeros(32, dtype=np.uint8), 255
    top = float(np.max(np.abs(x)))
    e = -125
    if top > 0:
        frac, power = math.frexp(top)                      # top = frac * 2^power, frac in [0.5, 1)
        e = min(125, max(-125, (power if frac >= 0.875 else power - 1) - 2))
    dist = np.abs(np.abs(x)[:, None] * 2.0 ** -e - STEPS)
    near = np.min(dist, axis=1, keepdims=True)
    codes = np.empty(32, dtype=np.uint8)
    for i in range(32):
        tied = np.nonzero(dist[i] == near[i])[0]
        codes[i] = next((c for c in tied if c % 2 == 0), tied[0])
    return codes | (np.signbit(x).astype(np.uint8) << 3), e + 127


def open_block(codes, biased):
    if biased == 255:
        return np.full(32, np.nan)
    return np.where(codes & 8, -1.0, 1.0) * STEPS[codes & 7] * 2.0 ** (int(biased) - 127)


def rounded(x):
    """Values that the cache stands for once x [..., head_dim] is stored."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(-1, 32)
    fine = np.all(np.isfinite(b), axis=1)
    frac, power = np.frexp(np.max(np.abs(np.where(fine[:, None], b, 0.0)), axis=1))
    e = np.clip(np.where(frac >= 0.875, power, power - 1) - 2, -125, 125)
    e = np.where(frac == 0, -125, e)
    dist = np.abs(np.abs(b)[:, :, None] * 2.0 ** -e[:, None, None].astype(np.float64) - STEPS)
    even, odd = dist[:, :, 0::2], dist[:, :, 1::2]
    code = np.where(even.min(-1) <= odd.min(-1), 2 * even.argmin(-1), 2 * odd.argmin(-1) + 1)
    y = np.copysign(STEPS[code] * 2.0 ** e[:, None].astype(np.float64), b)
    return np.where(fine[:, None], y, np.nan).reshape(x.shape)


def store(pool, k, v, slots):
    """Write tokens into pool (uint8 [pages][heads][17 * head_dim]); slots outside it are left out."""
    n_pages, heads, size = pool.shape
    dh = size // 17
    for r, slot in enumerate(slots):
        if not 0 <= slot < n_pages * PAGE:
            continue
        page, tok = int(slot) // PAGE, int(slot) % PAGE
        for h in range(heads):
            for value, x in enumerate((k, v)):
                for b in range(dh // 32):
                    codes, e = round_block(x[r, h, 32 * b:32 * b + 32])
                    at = value * 8 * dh + (b * PAGE + tok) * 16
                    pool[page, h, at:at + 16] = codes[0::2] | (codes[1::2] << 4)
                    pool[page, h, 16 * dh + (b * PAGE + tok) * 2 + value] = e


def read(pool, slots):
    """(keys, values) [len(slots)][heads][head_dim] of the pool."""
    n_pages, heads, size = pool.shape
    dh = size // 17
    out = np.empty((2, len(slots), heads, dh))
    for r, slot in enumerate(slots):
        block = pool[int(slot) // PAGE]
        tok = int(slot) % PAGE
        for h in range(heads):
            for value in range(2):
                for b in range(dh // 32):
                    at = value * 8 * dh + (b * PAGE + tok) * 16
                    byte = block[h, at:at + 16]
                    codes = np.stack((byte & 15, byte >> 4), axis=1).reshape(32)
                    out[value, r, h, 32 * b:32 * b + 32] = open_block(codes, block[h, 16 * dh + (b * PAGE + tok) * 2 + value])
    return out[0], out[1]


def extend(lens, new_lens, table, free, max_pages, n_pages, n_rows):
    """One iteration's tables.  table: list of page lists, free: stack (list), both changed in place unless refused.
    -> (lens, q_start, slots, positions, status)."""
    n = len(lens)
    held = [-(-x // PAGE) for x in lens]
    grown = [0 if a < 0 else x + a for x, a in zip(lens, new_lens)]
    refused = (list(lens), [0] * (n + 1), [-1] * n_rows, [-1] * n_rows)
    if (any(x < 0 or x > max_pages * PAGE or g > max_pages * PAGE for x, g in zip(lens, grown)) or
            sum(max(a, 0) for a in new_lens) > n_rows or len(free) + sum(h for h, a in zip(held, new_lens) if a < 0) > n_pages):
        return refused + (2,)
    back = [p for b in range(n) if new_lens[b] < 0 for p in table[b][:held[b]]]
    lack = [0 if a < 0 else -(-g // PAGE) - h for g, h, a in zip(grown, held, new_lens)]
    if sum(lack) > len(free) + len(back):
        return refused + (1,)
    free.extend(back)
    starts, slots, positions = [0], [], []
    for b in range(n):
        for _ in range(lack[b]):
            table[b][held[b]:held[b] + 1] = [free.pop()]
            held[b] += 1
        for pos in range(lens[b], grown[b]):
            slots.append(table[b][pos // PAGE] * PAGE + pos % PAGE)
            positions.append(pos)
        starts.append(len(slots))
    pad = [-1] * (n_rows - len(slots))
    return grown, starts, slots + pad, positions + pad, 0


def attention(q, k, v, scale):
    """Causal attention of q [rows][q_heads][dh], the last tokens of a sequence, over its keys and values [tokens][kv_heads][dh]:
    (out, lse, mean of |v| under the same weights - what a relative error of the weights can change)."""
    rows, hq, dh = q.shape
    n, hkv = k.shape[0], k.shape[1]
    out, lse, spread = np.zeros((rows, hq, dh)), np.full((rows, hq), -np.inf), np.zeros((rows, hq, dh))
    for i in range(rows):
        seen = n - rows + i + 1
        if seen <= 0:
            continue
        for h in range(hq):
            kk, vv = k[:seen, h // (hq // hkv)], v[:seen, h // (hq // hkv)]
            z = kk @ q[i, h] * scale
            m = np.max(z)
            p = np.exp(z - m)
            lse[i, h] = m + np.log(p.sum())
            out[i, h] = p @ vv / p.sum()
            spread[i, h] = p @ np.abs(vv) / p.sum()
    return out, lse, spread
