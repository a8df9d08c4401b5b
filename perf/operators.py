"""Performance cases of the 4-bit KV cache's operators: block tables and slot maps from request lengths, storing keys
and values, attention over the cache for single tokens and for many rows of a sequence.

The cache.  A page holds 16 tokens of one sequence; a sequence's pages are a row of its block table.  A key or value of a
head is kept in blocks of 32 dimensions: 4-bit codes (sign, and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) times a power of two
that the block shares (MXFP4).  Per page and KV head, head_dim * 17 bytes:
  keys    [head_dim / 32 blocks][16 tokens][16 bytes]     dimension 2 i of a block in the low half of byte i
  values  the same
  scales  [head_dim / 32 blocks][16 tokens][key, value]   biased exponents, 2^(e - 127); 255: the block is NaN

Kinds of case
  extend  one iteration's tables: `ended` sequences give their pages back, the others grow by new_lo..new_hi tokens
  append  `rows` tokens' keys and values stored through a slot map; some rows of the padded batch have no slot
  attend  causal attention of each sequence's last q_lo..q_hi tokens over its len_lo..len_hi cached ones (q_hi 0: over
          whole prompts, as many rows as tokens)
  step    the three in turn, as a decode iteration makes them
"""
import math
import random

import torch

own = False
PAGE = 16
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DEVICE = "cuda"


def listed():
    return [
        # a decode iteration's tables: 192 rollouts in flight get their next token's slot, 5 have just ended
        dict(name="extend_decode", kind="extend", seqs=192, old_lo=64, old_hi=4608, new_lo=1, new_hi=1, ended=5),
        # 384 prompts admitted at once
        dict(name="extend_prompts", kind="extend", seqs=384, old_lo=0, old_hi=0, new_lo=1, new_hi=1999, ended=0),
        # a decode iteration's new keys and values, 384 rollouts of the 8 B shape
        dict(name="append_decode", kind="append", rows=384, hkv=8, dh=128, dtype="bf16"),
        # a prefill pass's, as a projection that accumulates in fp32 leaves them
        dict(name="append_prompts_f32", kind="append", rows=32768, hkv=8, dh=128, dtype="f32"),
        # one interactive rollout of the small model: nothing but latency
        dict(name="attend_single", kind="attend", seqs=1, hq=14, hkv=2, dh=64, len_lo=331, len_hi=331, q_lo=1, q_hi=1),
        # the default workload's batch in the middle of a step
        dict(name="attend_mid", kind="attend", seqs=192, hq=32, hkv=8, dh=128, len_lo=576, len_hi=4608, q_lo=1, q_hi=1),
        # the routed-expert model's heads, the widest batch with the longest responses
        dict(name="attend_wide", kind="attend", seqs=384, hq=32, hkv=4, dh=128, len_lo=1152, len_hi=9216, q_lo=1, q_hi=1),
        # a few rollouts deep in the response tail: few rows, long contexts
        dict(name="attend_long", kind="attend", seqs=7, hq=32, hkv=8, dh=128, len_lo=4500, len_hi=32768, q_lo=1, q_hi=1),
        # a few drafted tokens of each rollout, checked at once
        dict(name="attend_drafts", kind="attend", seqs=61, hq=20, hkv=4, dh=64, len_lo=100, len_hi=2003, q_lo=1, q_hi=5),
        # whole prompts packed, ragged
        dict(name="attend_prompts", kind="attend", seqs=21, hq=32, hkv=8, dh=128, len_lo=1, len_hi=1999, q_lo=0, q_hi=0),
        # rollouts continued after a pause: a piece of each behind a long cached part
        dict(name="attend_chunks", kind="attend", seqs=3, hq=32, hkv=8, dh=128, len_lo=9001, len_hi=16384, q_lo=129, q_hi=300),
        # a whole decode iteration of the small model's heads
        dict(name="step_decode", kind="step", seqs=96, hq=14, hkv=2, dh=64, len_lo=257, len_hi=2304),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["extend", "append", "attend", "attend", "rows", "step"])
    if kind == "extend":
        seqs = _log(rng, 1, 400)
        if rng.random() < 0.5:
            return dict(kind=kind, seqs=seqs, old_lo=0, old_hi=_log(rng, 1, 9000), new_lo=0, new_hi=_log(rng, 1, 6), ended=rng.randint(0, seqs // 8))
        return dict(kind=kind, seqs=seqs, old_lo=0, old_hi=rng.choice([0, 700]), new_lo=0, new_hi=_log(rng, 20, 1900), ended=rng.randint(0, seqs // 8))
    hkv, group, dh = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.choice([32, 64, 128, 128])
    if kind == "append":
        return dict(kind=kind, rows=_log(rng, 1, 32000), hkv=hkv, dh=dh, dtype=rng.choice(["bf16", "f32"]))
    heads = dict(hq=hkv * group, hkv=hkv, dh=dh)
    # tokens of cache such that no case is larger than the largest listed one
    room = 384 * 5000 * 4 * 128 // (hkv * dh)
    if kind == "rows":
        whole = rng.random() < 0.5
        hi = _log(rng, 20, 2000 if whole else 12000)
        most = max(1, min(20, (1 << 27) // (heads["hq"] * hi * (hi if whole else 300))))
        q = rng.randint(6, 300)
        return dict(kind="attend", seqs=_log(rng, 1, most), **heads, len_lo=rng.choice([0, hi // 2]), len_hi=hi,
                    q_lo=0 if whole else q // 3, q_hi=0 if whole else q)
    hi = _log(rng, 1, 32768 if kind == "attend" else 4000)
    seqs = _log(rng, 1, max(1, min(384, room // hi, (1 << 30) // (heads["hq"] * hi))))
    if kind == "step":
        return dict(kind=kind, seqs=seqs, **heads, len_lo=rng.choice([1, (hi + 1) // 2]), len_hi=hi)
    q = rng.choice([1, 1, 2, 4])
    return dict(kind=kind, seqs=seqs, **heads, len_lo=rng.choice([0, hi // 2, hi]), len_hi=hi, q_lo=min(1, q - 1) if q > 1 else 1, q_hi=q)


# --- inputs ------------------------------------------------------------------------------------------------------------


def _ceil(a, b):
    return -(-a // b)


def _lengths(case):
    """Lengths in the cache and rows of each sequence, of a batch of this case (the same for every seed)."""
    r = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    n, q = [], []
    for _ in range(case["seqs"]):
        n.append(r.randint(case["len_lo"], case["len_hi"]))
        q.append(n[-1] if case.get("q_hi", 1) == 0 else r.randint(case.get("q_lo", 1), case.get("q_hi", 1)))
        if case["kind"] == "attend":
            q[-1] = min(q[-1], max(n[-1], 1))
    n[-1] = case["len_hi"]
    if case.get("q_hi", 1) == 0:
        q[-1] = n[-1]
    return n, q


def _grown(case):
    """Tokens held, and gained (-1: the sequence has ended), of each sequence of an `extend` case."""
    r = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    old = [r.randint(case["old_lo"], case["old_hi"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    for b in r.sample(range(case["seqs"]), case["ended"]):
        new[b] = -1
    return old, new


def _normal(shape, gen, channels=False):
    x = torch.randn(shape, generator=gen, device=DEVICE)
    if channels:  # keys have a few strong channels, the same for every token
        x *= torch.exp(0.5 * torch.randn((1,) + tuple(shape[1:]), generator=gen, device=DEVICE))
    return x


def _fill(pool, gen):
    """Keys and values of every token of the pool, some of them strong channels, a run of pages at a time."""
    n_pages, hkv, size = pool.shape
    dh = size // 17
    run = max(1, (1 << 26) // (PAGE * hkv * dh))
    for p in range(0, n_pages, run):
        n = min(run, n_pages - p)
        parts = []
        for key in (True, False):
            codes, scales, _ = _rounded(_normal((n * PAGE, hkv, dh), gen, key))
            parts.append((codes.view(n, PAGE, hkv, dh // 32, 16).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1), scales.view(n, PAGE, hkv, -1).permute(0, 2, 3, 1)))
        (k, ks), (v, vs) = parts
        pool[p : p + n] = torch.cat((k, v, torch.stack((ks, vs), -1).reshape(n, hkv, -1)), 2)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _tables(lens, spare, gen):
    """A block table of pages in no order, the pages that are free on a stack, and how many."""
    held = [_ceil(n, PAGE) for n in lens]
    n_pages = sum(held) + spare
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    cols = max(max(held), 1)
    at = torch.tensor([0] + held, device=DEVICE).cumsum(0)
    col = torch.arange(cols, device=DEVICE)
    rows = (at[:-1, None] + col).clamp(max=n_pages - 1)
    table = torch.where(col < torch.tensor(held, device=DEVICE)[:, None], order[rows], 0)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE)
    free[:spare] = order[n_pages - spare :]
    return table.contiguous(), free, _i32([spare])


def _widened(table, cols):
    return torch.cat((table, torch.zeros((table.shape[0], cols - table.shape[1]), dtype=torch.int32, device=DEVICE)), 1) if cols > table.shape[1] else table


def _plan(seqs, rows):
    """What april_cache_extend writes: lengths, free pages, first rows, slots, positions, status."""
    e = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device=DEVICE)  # noqa: E731
    return e(seqs), e(1), e(seqs + 1), e(rows, torch.int64), e(rows), e(1)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(kind=case["kind"])
    if case["kind"] == "extend":
        old, new = _grown(case)
        spare = sum(_ceil(o + max(n, 0), PAGE) - _ceil(o, PAGE) for o, n in zip(old, new)) + 3
        table, s["free"], s["top"] = _tables(old, spare, gen)
        s["table"] = _widened(table, max(_ceil(o + max(n, 0), PAGE) for o, n in zip(old, new)))
        rows = sum(max(n, 0) for n in new) + 5  # a padded batch
        s |= dict(lens=_i32(old), new=_i32(new), plan=_plan(len(old), rows), rows=rows)
        return s
    hkv, dh = case["hkv"], case["dh"]
    if case["kind"] == "append":
        rows = case["rows"]
        n_pages = _ceil(rows, PAGE) + 7
        s["pool"] = torch.zeros((n_pages, hkv, 17 * dh), dtype=torch.uint8, device=DEVICE)
        s["slots"] = torch.randperm(n_pages * PAGE, generator=gen, device=DEVICE)[:rows]
        s["slots"][rows - rows // 50 :] = -1  # a padded batch
        t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["k"], s["v"] = _normal((rows, hkv, dh), gen, True).to(t), _normal((rows, hkv, dh), gen).to(t)
        s["kv"], s["vv"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        return s
    lens, q = _lengths(case)
    if case["kind"] == "step":  # the token that this iteration adds is not in the cache yet
        table, s["free"], s["top"] = _tables(lens, len(lens) + 3, gen)
        s["table"] = _widened(table, _ceil(max(lens) + 1, PAGE))
        s |= dict(lens=_i32(lens), new=_i32([1] * len(lens)), plan=_plan(len(lens), len(lens)), rows=len(lens), max_len=max(lens) + 1)
        s["k"], s["v"] = _normal((len(lens), hkv, dh), gen, True).bfloat16(), _normal((len(lens), hkv, dh), gen).bfloat16()
        n_pages = s["free"].numel()
    else:
        s["table"], free, _ = _tables(lens, 3, gen)
        n_pages = free.numel()
        s |= dict(lens=_i32(lens), max_len=max(max(lens), 1))
    s["pool"] = torch.zeros((n_pages, hkv, 17 * dh), dtype=torch.uint8, device=DEVICE)
    _fill(s["pool"], gen)
    rows = sum(q)
    s["q"] = _normal((rows, case["hq"], dh), gen).bfloat16()
    s["q_start"] = None if case["kind"] == "step" or case["q_hi"] == case["q_lo"] == 1 else _i32([sum(q[:i]) for i in range(len(q) + 1)])
    s["max_q"] = max(q)
    s["out"] = torch.zeros((rows, case["hq"], dh), dtype=torch.bfloat16, device=DEVICE)
    s["lse"] = torch.zeros((rows, case["hq"]), dtype=torch.float32, device=DEVICE)
    return s


# --- the plain form ----------------------------------------------------------------------------------------------------


def _rounded(x):
    """Codes [..., dh / 32, 16] (two to a byte), biased exponents [..., dh / 32] and the values they stand for, of x [..., dh].

    A block's power of two is the one that brings its largest magnitude into [3.5, 7): the largest code, 6, is then off
    by no more than half a step of the next power of two's codes.  (Between 2^-125 and 2^125, so that every value is a normal
    number of bf16 and fp32.)  Codes round to nearest, ties to the even code.
    """
    x = x.float()
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    top = b.abs().amax(-1)
    e = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(min=2, max=252)
    bad = ~torch.isfinite(b).all(-1)
    e = torch.where(bad, 127, e)
    y = b * ((254 - e) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = torch.where(bad[..., None], 0, code + 8 * torch.signbit(b))
    value = _value_of(code.to(torch.uint8)) * (e << 23).view(torch.float32)[..., None]
    value = torch.where(bad[..., None], math.nan, value)
    codes = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    return codes, torch.where(bad, 255, e).to(torch.uint8), value.reshape(x.shape)


def _value_of(code):
    m = (code & 7).float()
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, 2 * m - 8))
    return torch.where(code >= 8, -v, v)


def _opened(pool, table):
    """Keys and values [sequence][KV head][token][dimension] in fp32 of the table's pages."""
    n_pages, hkv, size = pool.shape
    dh = size // 17
    pages = pool[table.long()]  # [sequence][page][head][bytes]
    s, p = table.shape
    pair = torch.arange(256, dtype=torch.uint8, device=pool.device)
    pair = torch.stack((_value_of(pair & 15), _value_of(pair >> 4)), -1)
    codes = pages[..., : 16 * dh].reshape(s, p, hkv, 2, dh // 32, PAGE, 16)
    scales = pages[..., 16 * dh :].reshape(s, p, hkv, dh // 32, PAGE, 2).permute(0, 1, 2, 5, 3, 4)
    factor = torch.where(scales == 255, math.nan, torch.ldexp(torch.ones((), device=pool.device), scales.int() - 127))
    x = pair.index_select(0, codes.reshape(-1).int()).reshape(s, p, hkv, 2, dh // 32, PAGE, 32) * factor[..., None]
    x = x.permute(3, 0, 2, 1, 5, 4, 6).reshape(2, s, hkv, p * PAGE, dh)
    return x[0], x[1]


def _attend(q, pool, table, lens, q_start, max_q, out, lse):
    seqs, (rows, hq, dh), hkv = lens.numel(), q.shape, pool.shape[1]
    first = torch.arange(seqs + 1, device=q.device) if q_start is None else q_start.long()
    count = first[1:] - first[:-1]
    i = torch.arange(max_q, device=q.device)
    row = (first[:-1, None] + i).clamp(max=rows - 1)  # [sequence][its row]
    mine = i < count[:, None]
    k, v = _opened(pool, table)
    x = q.float()[row].reshape(seqs, max_q, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, -1, dh)
    score = torch.matmul(x, k.transpose(-1, -2)).reshape(seqs, hkv, hq // hkv, max_q, -1) / math.sqrt(dh)
    t = torch.arange(k.shape[2], device=q.device)
    seen = t < (lens.long() - count)[:, None, None] + i[:, None] + 1  # [sequence][its row][token]
    seen &= t < lens[:, None, None]
    score = torch.where(seen[:, None, None], score, -math.inf)
    m = score.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(score - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(seqs, hkv, -1, p.shape[-1]), v).reshape(p.shape[:-1] + (dh,)) / torch.where(total == 0, 1.0, total)
    l = (torch.log(total) + m)[..., 0]
    o, l = o.permute(0, 3, 1, 2, 4).reshape(seqs, max_q, hq, dh), l.permute(0, 3, 1, 2).reshape(seqs, max_q, hq)
    out[row[mine]] = o[mine].to(out.dtype)
    lse[row[mine]] = l[mine]
    return out, lse


def _append(pool, k, v, slots, kv=None, vv=None):
    """Rows without a slot are left out.  `kv`, `vv`: the values that the cache then stands for."""
    n_pages, hkv, size = pool.shape
    dh = size // 17
    there = (slots >= 0) & (slots < n_pages * PAGE)
    page, t = slots[there] // PAGE, slots[there] % PAGE
    for x, at, to in ((k, 0, kv), (v, 1, vv)):
        codes, scales, value = _rounded(x[there])
        pool[..., 8 * dh * at : 8 * dh * (at + 1)].view(n_pages, hkv, dh // 32, PAGE, 16)[page, :, :, t] = codes
        pool[..., 16 * dh :].view(n_pages, hkv, dh // 32, PAGE, 2)[page, :, :, t, at] = scales
        if to is not None:
            to[there] = value.to(to.dtype)


def _extend(lens, new, table, free, top, rows, plan):
    """Pages of the ended sequences go onto the stack, in order; then each sequence takes what it lacks from its top."""
    seqs, cols = table.shape
    lens64, top64 = lens.long(), top.long()
    held = (lens64 + PAGE - 1) // PAGE
    col = torch.arange(cols, device=lens.device)
    gone = (new < 0)[:, None] & (col < held[:, None])
    free[(top64 + gone.reshape(-1).cumsum(0) - 1).reshape(seqs, cols)[gone]] = table[gone]
    have = top64 + gone.sum()
    add = new.long().clamp(min=0)
    after = torch.where(new < 0, 0, lens64 + add)
    lack = ((after + PAGE - 1) // PAGE - held).clamp(min=0)
    taken = lack.cumsum(0) - lack  # pages that the sequences before take
    grows = (col >= held[:, None]) & (col < (held + lack)[:, None])
    table[grows] = free[have - 1 - (taken[:, None] + col - held[:, None])[grows]]
    to_lens, to_top, q_start, slots, positions, status = plan
    to_lens.copy_(after)
    to_top.copy_(have - lack.sum())
    q_start[0] = 0
    q_start[1:] = add.cumsum(0)
    r = torch.arange(rows, device=lens.device)
    b = torch.searchsorted(q_start, r, right=True) - 1
    mine = r < q_start[-1]
    b = b.clamp(max=seqs - 1)
    pos = lens64[b] + r - q_start[b]
    positions.copy_(torch.where(mine, pos, -1))
    slots.copy_(torch.where(mine, table[b, (pos // PAGE).clamp(max=cols - 1)] * PAGE + pos % PAGE, -1))
    status.zero_()
    return plan


def run(s):
    if own:
        import paper_2509_18521_amd as ap

        if s["kind"] == "extend":
            ap.april_cache_extend(s["lens"], s["new"], s["table"], s["free"], s["top"], s["rows"], out=s["plan"])
            return s["plan"], s["table"]
        if s["kind"] == "append":
            ap.april_cache_append(s["pool"], s["k"], s["v"], s["slots"], k_values=s["kv"], v_values=s["vv"])
            return s["kv"], s["vv"]
        lens = s["lens"]
        if s["kind"] == "step":
            lens, _, _, slots, _, _ = ap.april_cache_extend(lens, s["new"], s["table"], s["free"], s["top"], s["rows"], out=s["plan"])
            ap.april_cache_append(s["pool"], s["k"], s["v"], slots)
        ap.april_cache_attention(s["q"], s["pool"], s["table"], lens, s["max_len"], q_start=s["q_start"], max_q=s["max_q"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    if s["kind"] == "extend":
        return _extend(s["lens"], s["new"], s["table"], s["free"], s["top"], s["rows"], s["plan"]), s["table"]
    if s["kind"] == "append":
        _append(s["pool"], s["k"], s["v"], s["slots"], s["kv"], s["vv"])
        return s["kv"], s["vv"]
    lens = s["lens"]
    if s["kind"] == "step":
        lens, _, _, slots, _, _ = _extend(lens, s["new"], s["table"], s["free"], s["top"], s["rows"], s["plan"])
        _append(s["pool"], s["k"], s["v"], slots)
    return _attend(s["q"], s["pool"], s["table"], lens, s["q_start"], s["max_q"], s["out"], s["lse"])


def work(case):
    """Each input read once, each output written once; attention's products over the tokens that a row sees."""
    if case["kind"] == "extend":
        old, new = _grown(case)
        pages = sum(abs(_ceil(o + n, PAGE) - _ceil(o, PAGE)) if n >= 0 else _ceil(o, PAGE) for o, n in zip(old, new))
        rows = sum(max(n, 0) for n in new)
        return dict(bytes=16 * len(old) + 8 * pages + 12 * rows, flops=0)
    kept = case["hkv"] * case["dh"] * 17 / 16  # a token's bytes in the cache
    if case["kind"] == "append":
        e = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] - case["rows"] // 50
        return dict(bytes=n * (2 * case["hkv"] * case["dh"] * e * 2 + kept + 8), flops=0)
    lens, q = _lengths(case)
    tokens, rows, seen = sum(lens), sum(q), sum(sum(n - c + i + 1 for i in range(c)) if n >= c else 0 for n, c in zip(lens, q))
    pages = sum(_ceil(n, PAGE) for n in lens)
    b = tokens * kept + 4 * pages + rows * case["hq"] * (4 * case["dh"] + 4)
    if case["kind"] == "step":
        b += rows * (4 * case["hkv"] * case["dh"] + kept + 40)
        seen += rows
    return dict(bytes=b, flops=4 * seen * case["hq"] * case["dh"])


# --- in 64 bits, from the definitions, a sequence at a time -------------------------------------------------------------


def _exact_values(x):
    """What blocks of 32 of x are rounded to: the power of two from the largest magnitude's fraction and exponent, the nearest
    of the even codes and the nearest of the odd ones, the nearer of the two (the even one on a tie)."""
    b = x.double().reshape(-1, 32)
    frac, power = torch.frexp(b.abs().amax(1))
    e = torch.where(frac >= 0.875, power, power - 1) - 2
    one = torch.ldexp(torch.ones_like(frac), e.clamp(min=-125, max=125))[:, None]
    even, odd = (torch.tensor(STEPS[i::2], dtype=torch.float64, device=x.device) for i in (0, 1))
    a = b.abs() / one
    de, do = ((a[..., None] - g).abs() for g in (even, odd))
    near_e, near_o = even[de.argmin(-1)], odd[do.argmin(-1)]
    return (torch.where(de.amin(-1) <= do.amin(-1), near_e, near_o) * torch.sign(b) * one).reshape(x.shape)


def _exact_page_values(block):
    """Keys and values [2][page][token][dh] of one head's pages [page][17 dh bytes]."""
    dh, n = block.shape[1] // 17, block.shape[0]
    codes = block[:, : 16 * dh].reshape(n, 2, dh // 32, PAGE, 16).int()
    nib = torch.stack((codes & 15, codes >> 4), -1).reshape(n, 2, dh // 32, PAGE, 32)
    steps = torch.tensor(STEPS + tuple(-v for v in STEPS), dtype=torch.float64, device=block.device)
    e = block[:, 16 * dh :].reshape(n, dh // 32, PAGE, 2).permute(0, 3, 1, 2).double() - 127
    return (steps[nib] * torch.exp2(e)[..., None]).permute(1, 0, 3, 2, 4).reshape(2, n, PAGE, dh)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "extend":
        lens, new, free, top = s["lens"].tolist(), s["new"].tolist(), s["free"].tolist(), int(s["top"])
        table = [r[: _ceil(n, PAGE)] for r, n in zip(s["table"].tolist(), lens)]
        stack = free[:top] + [p for r, n in zip(table, new) if n < 0 for p in r]
        whole, slots, positions, starts = s["table"].cpu(), [], [], [0]
        for b, (r, n, m) in enumerate(zip(table, lens, new)):
            m = max(m, 0)
            while len(r) * PAGE < n + m and new[b] >= 0:
                r.append(stack.pop())
                whole[b, len(r) - 1] = r[-1]
            slots += [r[(n + i) // PAGE] * PAGE + (n + i) % PAGE for i in range(m)]
            positions += range(n, n + m)
            starts.append(starts[-1] + m)
        pad = [-1] * (s["rows"] - len(slots))
        i64 = lambda v: torch.tensor(v, dtype=torch.int64)  # noqa: E731
        after = [0 if m < 0 else n + m for n, m in zip(lens, new)]
        return (i64(after), i64([len(stack)]), i64(starts), i64(slots + pad), i64(positions + pad), i64([0])), whole
    if case["kind"] == "append":
        got = []
        for x in (s["k"], s["v"]):
            y = torch.zeros_like(x, dtype=torch.float64)
            y[s["slots"] >= 0] = _exact_values(x[s["slots"] >= 0])
            got.append(y)
        return tuple(got)
    lens, q = _lengths(case)
    dh, hkv = case["dh"], case["hkv"]
    group = case["hq"] // hkv
    out, lse, row = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE), torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE), 0
    if case["kind"] == "step":
        k_new, v_new = _exact_values(s["k"]), _exact_values(s["v"])
    for b, (n, c) in enumerate(zip(lens, q)):
        pages = s["table"][b, : _ceil(n, PAGE)].long()
        for h in range(hkv):
            k, v = _exact_page_values(s["pool"][pages, h]).reshape(2, -1, dh)[:, :n]
            if case["kind"] == "step":
                k, v = torch.cat((k, k_new[b : b + 1, h])), torch.cat((v, v_new[b : b + 1, h]))
            total = k.shape[0]
            if c == 0 or total == 0:
                continue
            x = s["q"][row : row + c, h * group : (h + 1) * group].double()
            z = torch.matmul(x.reshape(-1, dh), k.T).reshape(c, group, total) / math.sqrt(dh)
            sees = torch.arange(total, device=DEVICE) <= total - c + torch.arange(c, device=DEVICE)[:, None]
            z = z.masked_fill(~sees[:, None], -math.inf)
            lse[row : row + c, h * group : (h + 1) * group] = torch.logsumexp(z, -1)
            out[row : row + c, h * group : (h + 1) * group] = torch.nan_to_num(torch.softmax(z, -1)).reshape(-1, total).matmul(v).reshape(c, group, dh)
        row += c
    return out, lse
