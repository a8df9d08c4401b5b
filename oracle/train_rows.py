"""The scoring and training operators in 64 bits, from their definitions: log-probabilities with entropy and alternatives, the embedding,
tokens' rows in their experts' batches, and their gradients.  Plain numpy, a row at a time."""
from __future__ import annotations

import numpy as np


def logprobs(logits, tokens, temperature=1.0, top=0):
    """(logprob, entropy, lse, top logprobs, top ids) of logits [n, vocab]; a token below zero: zeros, ids -1; one of vocab or more: a logprob of NaN.  A row with
    a NaN, +infinity or nothing but -infinity: NaN, ids -1."""
    n, vocab = logits.shape
    lp, ent, lse = np.zeros(n), np.zeros(n), np.zeros(n)
    best, ids = np.zeros((n, top)), np.full((n, top), -1, dtype=np.int64)
    for r in range(n):
        if tokens[r] < 0:
            continue
        row = np.asarray(logits[r], dtype=np.float64)
        m = np.max(row)
        if not np.isfinite(m):
            lp[r] = ent[r] = np.nan
            lse[r] = -np.inf if m == -np.inf else np.nan
            best[r] = np.nan
            continue
        y = (row - m) / temperature
        s = np.sum(np.exp(y))
        logp = y - np.log(s)
        p = np.exp(logp)
        ent[r] = -np.sum(p[p > 0] * logp[p > 0])
        lse[r] = m / temperature + np.log(s)
        lp[r] = logp[tokens[r]] if tokens[r] < vocab else np.nan
        order = np.lexsort((np.arange(vocab), -row))[:top]
        ids[r], best[r] = order, logp[order]
    return lp, ent, lse, best, ids


def logprobs_grad(logits, tokens, temperature, g=None, h=None, z=None):
    """(gradient of the logits, sum of its terms' magnitudes) for gradients of logprob, entropy and lse."""
    n, vocab = logits.shape
    out, size = np.zeros((n, vocab)), np.zeros((n, vocab))
    for r in range(n):
        if tokens[r] < 0:
            continue
        y = np.asarray(logits[r], dtype=np.float64) / temperature
        if not np.isfinite(np.max(y)):
            out[r] = np.nan
            continue
        y = y - np.max(y)
        logp = y - np.log(np.sum(np.exp(y)))
        p = np.exp(logp)
        gr, hr, zr = (0.0 if v is None else float(v[r]) for v in (g, h, z))
        plogp = np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0)
        ent = -np.sum(plogp)
        out[r] = (zr - gr) * p - hr * (plogp + p * ent)
        size[r] = (abs(zr) + abs(gr)) * p + abs(hr) * (np.abs(plogp) + p * ent)
        if tokens[r] < vocab:
            out[r, tokens[r]] += gr
            size[r, tokens[r]] += abs(gr)
        else:
            out[r] = np.nan
    return out / temperature, size / temperature


def embed(table, tokens, scale=1.0):
    out = np.zeros((len(tokens), table.shape[1]))
    for r, t in enumerate(tokens):
        if t >= len(table):
            out[r] = np.nan
        elif t >= 0:
            out[r] = scale * table[t]
    return out


def embed_grad(grad_out, tokens, vocab, scale=1.0, start=None):
    """(gradient of the table, sum of its terms' magnitudes, rows of each token); start: what it is added to."""
    out = np.zeros((vocab, grad_out.shape[1])) if start is None else np.array(start, dtype=np.float64)
    size, rows = np.abs(out), np.zeros(vocab, dtype=np.int64)
    for r, t in enumerate(tokens):
        if 0 <= t < vocab:
            out[t] += scale * grad_out[r]
            size[t] += np.abs(scale * grad_out[r])
            rows[t] += 1
    return out, size, rows


def packed_rows(n, n_experts, align):
    return (n + min(n_experts, n) * (align - 1)) // align * align


def expert_sort(ids, n_experts, align=1):
    """(starts, source, position)."""
    flat = ids.reshape(-1)
    source, position, starts = np.full(packed_rows(flat.size, n_experts, align), -1), np.full(flat.size, -1), [0]
    for e in range(n_experts):
        at = starts[-1]
        for a, x in enumerate(flat):
            if x == e:
                source[at], position[a] = a, at
                at += 1
        starts.append(-(-at // align) * align)
    return np.array(starts), source, position.reshape(ids.shape)


def expert_gather(x, source, k):
    out = np.zeros((len(source), x.shape[1]))
    for p, a in enumerate(source):
        if a >= 0:
            out[p] = x[a // k]
    return out


def expert_combine(packed, position, weights=None):
    """(sums, sums of the terms' magnitudes)."""
    out, size = np.zeros((len(position), packed.shape[1])), np.zeros((len(position), packed.shape[1]))
    for r, places in enumerate(position):
        for j, p in enumerate(places):
            if p >= 0:
                v = packed[p] * (1.0 if weights is None else weights[r, j])
                out[r] += v
                size[r] += np.abs(v)
    return out, size


def expert_combine_grad(grad_out, packed, source, position, weights=None):
    """(gradient of packed, of the weights, sums of the latter's terms' magnitudes)."""
    k = position.shape[1]
    of_packed, of_weights, size = np.zeros(packed.shape), np.zeros(position.shape), np.zeros(position.shape)
    for p, a in enumerate(source):
        if a >= 0:
            r, j = a // k, a % k
            of_packed[p] = grad_out[r] * (1.0 if weights is None else weights[r, j])
            of_weights[r, j] = np.sum(grad_out[r] * packed[p])
            size[r, j] = np.sum(np.abs(grad_out[r] * packed[p]))
    return of_packed, of_weights, size
