"""Performance cases of the operators that score rollouts and train on them, where a row is chosen by an index: the
log-probability of a given token with the entropy and the most likely alternatives, a token's row of the embedding, a token's
rows in its experts' batches; each with its gradient.

Kinds of case
  score    log softmax(logits / temperature)[token] of each row, its entropy and its `top` largest (descending, ties by
           the lower index); rows of token -1 are padding: zeros, ids -1
  policy   the first two and the gradient of the logits, as a policy-gradient step asks for it
  embed    rows of the embedding, scaled; padding gives zeros
  learn    the same and the embedding's gradient: the sum of the gradients of a token's rows (tokens as skewed as words are)
  experts  tokens' assignments sorted by expert (`align`: each expert's rows begin at a multiple of it, rows between are
           zeros), the tokens' rows gathered in that order, and what the experts made of them summed by the router's weights
  route    the same and its gradients: of the tokens' rows, of the experts' results, of the weights
"""
import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one interactive rollout's next token with its alternatives: nothing but latency
        dict(name="score_single", kind="score", rows=1, vocab=151936, pad=0, dtype="f32", top=20, temperature=1.0, masked=0),
        # a decode iteration of the default workload: logits as the engine leaves them
        dict(name="score_decode", kind="score", rows=192, vocab=151936, pad=0, dtype="f32", top=5, temperature=1.0, masked=0),
        # rollouts scored under another policy (a reference model, the next policy's first pass)
        dict(name="score_rollouts", kind="score", rows=8192, vocab=128256, pad=0, dtype="bf16", top=0, temperature=1.0, masked=0),
        # an odd vocabulary in wider rows, half of the positions prompts or padding, the widest list of alternatives
        dict(name="score_odd", kind="score", rows=2777, vocab=32003, pad=61, dtype="bf16", top=64, temperature=0.6, masked=50),
        # the training step at the small and the default model's vocabulary
        dict(name="policy_train", kind="policy", rows=16384, vocab=151936, pad=0, dtype="bf16", top=0, temperature=1.0, masked=25),
        # the smallest model's, in fp32
        dict(name="policy_tiny", kind="policy", rows=768, vocab=512, pad=0, dtype="f32", top=0, temperature=0.8, masked=10),
        # a decode iteration's rows into an fp32 residual stream
        dict(name="embed_decode", kind="embed", rows=192, vocab=151936, d=2560, dtype="bf16", out="f32", scale=1.0, masked=0),
        # a training pass over packed rollouts of the default model
        dict(name="learn_train", kind="learn", rows=32768, vocab=151936, d=2560, dtype="bf16", out="bf16", scale=1.0, masked=10),
        # an odd width and vocabulary in fp32, scaled as some models do
        dict(name="learn_odd", kind="learn", rows=5001, vocab=32003, d=1037, dtype="f32", out="f32", scale=32.2, masked=0),
        # a decode iteration of the routed-expert model
        dict(name="experts_decode", kind="experts", rows=384, experts=128, k=8, d=2048, dtype="bf16", align=64),
        # a prefill pass of it
        dict(name="experts_prompts", kind="experts", rows=13900, experts=128, k=8, d=2048, dtype="bf16", align=128),
        # a training pass, some tokens' experts elsewhere
        dict(name="route_train", kind="route", rows=16384, experts=128, k=8, d=2048, dtype="bf16", align=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["score", "score", "policy", "embed", "learn", "experts", "route"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("score", "policy"):
        vocab = _log(rng, 300, 160000)
        rows = _log(rng, 1, min(16384, (1 << 29) // vocab))
        top = rng.choice([0, 1, 5, 20, 64]) if kind == "score" else 0
        return dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, 0, rng.randint(1, 64)]), dtype=dtype, top=top,
                    temperature=rng.choice([1.0, 1.0, 0.6, 1.3]), masked=rng.choice([0, 0, rng.randint(5, 70)]))
    d = rng.choice([8 * _log(rng, 8, 1000), _log(rng, 50, 6000)])
    if kind in ("embed", "learn"):
        vocab = _log(rng, 300, min(160000, (1 << 28) // d))
        return dict(kind=kind, rows=_log(rng, 1, min(32768, (1 << 26) // d)), vocab=vocab, d=d, dtype=dtype, out=rng.choice([dtype, "f32"]),
                    scale=rng.choice([1.0, round(math.sqrt(d), 2)]), masked=rng.choice([0, 0, 20]))
    experts = _log(rng, 4, 256)
    k = rng.randint(1, min(experts, 10))
    return dict(kind=kind, rows=_log(rng, 1, min(16384, (1 << 28) // (d * k))), experts=experts, k=k, d=d, dtype=dtype, align=rng.choice([1, 8, 16, 64, 128]))


# --- inputs ------------------------------------------------------------------------------------------------------------


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _rand(gen, *shape):
    return torch.rand(shape, generator=gen, device=DEVICE)


def _packed_rows(case):
    """Rows that hold every assignment whatever the experts' shares are."""
    n, a = case["rows"] * case["k"], case["align"]
    return (n + min(case["experts"], n) * (a - 1)) // a * a


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    kind, rows = case["kind"], case["rows"]
    s = dict(kind=kind)
    if kind in ("score", "policy"):
        vocab, t = case["vocab"], TYPES[case["dtype"]]
        whole = torch.empty((rows, vocab + case["pad"]), dtype=t, device=DEVICE)
        tokens = torch.randint(vocab, (rows,), generator=gen, device=DEVICE)
        for r in range(0, rows, 2048):  # a trained model's logits: a wide bulk, and some probability at the token that was drawn
            part = whole[r : r + 2048]
            part.copy_(2.5 * _randn(gen, *part.shape))
            at = tokens[r : r + 2048, None]
            part.scatter_(1, at, (part.gather(1, at).float() + 12 * _rand(gen, part.shape[0], 1)).to(t))
        tokens[torch.randperm(rows, generator=gen, device=DEVICE)[: rows * case["masked"] // 100]] = -1
        s |= dict(logits=whole[:, :vocab], tokens=tokens, temperature=case["temperature"], top=case["top"])
        if kind == "policy":
            s |= dict(g_logprob=_randn(gen, rows), g_entropy=0.01 * (1 + _rand(gen, rows)))
        return s
    d = case["d"]
    if kind in ("embed", "learn"):
        vocab = case["vocab"]
        rank = torch.exp(_rand(gen, rows) * math.log(vocab)).long().clamp(max=vocab) - 1  # a word's frequency falls with its rank
        tokens = torch.randperm(vocab, generator=gen, device=DEVICE)[rank]
        tokens[torch.randperm(rows, generator=gen, device=DEVICE)[: rows * case["masked"] // 100]] = -1
        s |= dict(table=_randn(gen, vocab, d).to(TYPES[case["dtype"]]), tokens=tokens, scale=case["scale"], out=TYPES[case["out"]])
        if kind == "learn":
            s["grad"] = _randn(gen, rows, d).to(s["out"])
        return s
    t, k, e = TYPES[case["dtype"]], case["k"], case["experts"]
    liking = _randn(gen, rows, e) + 0.7 * _randn(gen, 1, e)  # some experts are asked for more than others
    w, ids = torch.topk(torch.softmax(liking, 1), k)
    if kind == "route":  # a share of the experts lies on another GPU
        ids = torch.where(ids >= e - e // 8, -1, ids)
    m = _packed_rows(case)
    s |= dict(x=_randn(gen, rows, d).to(t), ids=ids.int(), weights=(w / w.sum(1, keepdim=True)).contiguous(), experts=e, align=case["align"], packed=m, y=_randn(gen, m, d).to(t))
    if kind == "route":
        s |= dict(g_packed=_randn(gen, m, d).to(t), g_out=_randn(gen, rows, d).to(t))
    return s


# --- the plain form ----------------------------------------------------------------------------------------------------


def _softmax_parts(s):
    """Scaled logits, exponentials, their sum, log of the sum of exponentials, entropy, the token's log-probability."""
    there = s["tokens"] >= 0
    x = s["logits"].float() / s["temperature"]
    m = x.amax(1, keepdim=True)
    y = x - m
    e = torch.exp(y)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    entropy = (log_total - (e * y).sum(1, keepdim=True) / total)[:, 0]
    lse = (m + log_total)[:, 0]
    at = s["tokens"].clamp(min=0)[:, None]
    logprob = (y.gather(1, at) - log_total)[:, 0]
    return there, x, y, e, total, log_total, lse, torch.where(there, entropy, 0.0), torch.where(there, logprob, 0.0), at


def _score(s):
    there, x, _, _, _, _, lse, entropy, logprob, _ = _softmax_parts(s)
    if s["top"] == 0:
        return logprob, entropy
    bits = (s["logits"].float() + 0.0).view(torch.int32)  # order of floats as order of integers; then the lower index first
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (bits << 32) | (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
    ids = 0x7FFFFFFF - (torch.topk(key, s["top"], dim=1).values & 0x7FFFFFFF)
    best = x.gather(1, ids) - lse[:, None]
    return logprob, entropy, torch.where(there[:, None], best, 0.0), torch.where(there[:, None], ids, -1).int()


def _policy(s):
    there, _, y, e, total, log_total, _, entropy, logprob, at = _softmax_parts(s)
    g, h = (torch.where(there, s[n], 0.0)[:, None] / s["temperature"] for n in ("g_logprob", "g_entropy"))
    p = e / total
    grad = -p * (g + h * (y - log_total + entropy[:, None]))
    grad.scatter_add_(1, at, g)
    return logprob, entropy, grad.to(s["logits"].dtype)


def _embed(s):
    there = (s["tokens"] >= 0)[:, None]
    return torch.where(there, s["table"][s["tokens"].clamp(min=0)].float() * s["scale"], 0.0).to(s["out"])


def _learn(s):
    there = s["tokens"] >= 0
    grad = torch.zeros(s["table"].shape, dtype=torch.float32, device=DEVICE)
    grad.index_add_(0, s["tokens"][there], s["grad"][there].float())
    return _embed(s), (grad * s["scale"]).to(s["table"].dtype)


def _sorted(s):
    """First packed row of each expert, the assignment of each packed row, the packed row of each assignment."""
    ids, e, align = s["ids"], s["experts"], s["align"]
    flat = ids.reshape(-1).long()
    there = flat >= 0
    key = torch.where(there, flat, e)
    order = torch.argsort(key, stable=True)
    count = torch.bincount(key, minlength=e + 1)[:e]
    room = (count + align - 1) // align * align
    starts = torch.cat((room.new_zeros(1), room.cumsum(0)))
    before = torch.cat((count.new_zeros(1), count.cumsum(0)))
    row = starts[key[order]] + torch.arange(flat.numel(), device=DEVICE) - before[key[order]]
    position = torch.full_like(flat, -1)
    position[order] = torch.where(there[order], row, -1)
    source = torch.full((s["packed"] + 1,), -1, dtype=torch.int64, device=DEVICE)
    source[torch.where(position >= 0, position, s["packed"])] = torch.arange(flat.numel(), device=DEVICE)
    return starts.int(), source[: s["packed"]].int(), position.reshape(ids.shape).int()


def _back(y, position, weights):
    """Sums of the packed rows of each token, in fp32."""
    rows = torch.where((position >= 0)[..., None], y[position.clamp(min=0).long()].float(), 0.0)
    return (rows if weights is None else rows * weights[..., None]).sum(1)


def _experts(s):
    starts, source, position = _sorted(s)
    k = s["ids"].shape[1]
    there = (source >= 0)[:, None]
    token = torch.div(source.clamp(min=0), k, rounding_mode="floor").long()
    packed = torch.where(there, s["x"][token], 0)
    out = _back(s["y"], position, s["weights"]).to(s["x"].dtype)
    if s["kind"] == "experts":
        return starts, source, position, packed, out
    g_x = _back(s["g_packed"], position, None).to(s["x"].dtype)
    g = s["g_out"].float()
    g_y = torch.where(there, g[token] * s["weights"].reshape(-1)[source.clamp(min=0).long()][:, None], 0.0).to(s["y"].dtype)
    g_w = (torch.where((position >= 0)[..., None], s["y"][position.clamp(min=0).long()].float(), 0.0) * g[:, None]).sum(2)
    return starts, source, position, packed, out, g_x, g_y, g_w


def run(s):
    kind = s["kind"]
    if own:
        import paper_2509_18521_amd as ap

        if kind == "score":
            got = ap.april_logprobs(s["logits"], s["tokens"], temperature=s["temperature"], entropy=True, top=s["top"])
            return (got.logprob, got.entropy) if s["top"] == 0 else (got.logprob, got.entropy, got.top_logprobs, got.top_ids)
        if kind == "policy":
            leaf = s["logits"].detach().requires_grad_()
            got = ap.april_logprobs(leaf, s["tokens"], temperature=s["temperature"], entropy=True)
            (grad,) = torch.autograd.grad((got.logprob, got.entropy), leaf, (s["g_logprob"], s["g_entropy"]))
            return got.logprob.detach(), got.entropy.detach(), grad
        if kind == "embed":
            return ap.april_embed(s["table"], s["tokens"], scale=s["scale"], dtype=s["out"])
        if kind == "learn":
            leaf = s["table"].detach().requires_grad_()
            out = ap.april_embed(leaf, s["tokens"], scale=s["scale"], dtype=s["out"])
            (grad,) = torch.autograd.grad(out, leaf, s["grad"])
            return out.detach(), grad
        rows = ap.april_expert_sort(s["ids"], s["experts"], align=s["align"])
        if kind == "experts":
            packed = ap.april_expert_gather(s["x"], rows)
            return rows.starts, rows.source, rows.position, packed, ap.april_expert_combine(s["y"], rows, s["weights"])
        x, y, w = (s[n].detach().requires_grad_() for n in ("x", "y", "weights"))
        packed = ap.april_expert_gather(x, rows)
        out = ap.april_expert_combine(y, rows, w)
        grads = torch.autograd.grad((packed, out), (x, y, w), (s["g_packed"], s["g_out"]))
        return (rows.starts, rows.source, rows.position, packed.detach(), out.detach()) + grads
    if kind == "score":
        return _score(s)
    if kind == "policy":
        return _policy(s)
    if kind == "embed":
        return _embed(s)
    return _learn(s) if kind == "learn" else _experts(s)


def work(case):
    """Each input read once, each output written once (rows of padding: not read, but written where they are outputs)."""
    kind, rows, e = case["kind"], case["rows"], 2 if case["dtype"] == "bf16" else 4
    if kind in ("score", "policy"):
        vocab = case["vocab"]
        live = rows - rows * case["masked"] // 100
        b = live * vocab * e + rows * (8 + 8 + 8 * case["top"])
        if kind == "policy":
            b += rows * vocab * e + 8 * rows
        return dict(bytes=b, flops=live * vocab * (5 if kind == "score" else 10))
    d = case["d"]
    if kind in ("embed", "learn"):
        o = 2 if case["out"] == "bf16" else 4
        live = rows - rows * case["masked"] // 100
        b = min(live, case["vocab"]) * d * e + rows * (d * o + 8)
        if kind == "learn":
            b += live * d * o + case["vocab"] * d * e
        return dict(bytes=b, flops=rows * d * (1 if kind == "embed" else 2))
    n, m = rows * case["k"], _packed_rows(case)
    b = 4 * (2 * n + m + case["experts"] + 1) + rows * d * e + m * d * e + n * d * e + 4 * n + rows * d * e
    if kind == "route":  # gradients of the packed rows and of the sums, in; of x, y and the weights, out
        b += n * d * e + rows * d * e + rows * d * e + m * d * e + 4 * n
    return dict(bytes=b, flops=n * d * (2 if kind == "experts" else 6))


# --- in 64 bits, from the definitions ----------------------------------------------------------------------------------


def _exact_logits(case, s):
    rows, vocab = s["logits"].shape
    top = case["top"]
    logprob, entropy = (torch.zeros(rows, dtype=torch.float64, device=DEVICE) for _ in range(2))
    best = torch.zeros((rows, top), dtype=torch.float64, device=DEVICE)
    ids = torch.full((rows, top), -1, dtype=torch.int64, device=DEVICE)
    grad = torch.zeros((rows, vocab), dtype=torch.float64, device=DEVICE) if case["kind"] == "policy" else None
    per = max(1, (1 << 27) // vocab)
    live = torch.nonzero(s["tokens"] >= 0)[:, 0]
    for r in range(0, live.numel(), per):
        at = live[r : r + per]
        logp = torch.log_softmax(s["logits"][at].double() / case["temperature"], 1)
        p = torch.exp(logp)
        h = -(p * logp).sum(1)
        token = s["tokens"][at]
        one = torch.arange(at.numel(), device=DEVICE)
        logprob[at], entropy[at] = logp[one, token], h
        if grad is not None:
            z = p * -(s["g_logprob"][at].double()[:, None] + s["g_entropy"][at].double()[:, None] * (logp + h[:, None]))
            z[one, token] += s["g_logprob"][at].double()
            grad[at] = z / case["temperature"]
        if top:  # everything that is no less than the last of them, put in order on the host
            raw = s["logits"][at].double()
            row, col = torch.nonzero(raw >= torch.topk(raw, top, dim=1).values[:, -1:], as_tuple=True)
            row, col, v = row.cpu().numpy(), col.cpu().numpy(), raw[row, col].cpu().numpy()
            order = np.lexsort((col, -v, row))
            row, col = row[order], col[order]
            first = np.searchsorted(row, np.arange(at.numel()))
            col = torch.from_numpy(col[first[:, None] + np.arange(top)]).to(DEVICE)
            ids[at], best[at] = col, logp.gather(1, col)
    if case["kind"] == "policy":
        return logprob, entropy, grad
    return (logprob, entropy, best, ids) if top else (logprob, entropy)


def _exact_experts(case, s):
    ids, k, align, m = s["ids"].cpu().numpy(), case["k"], case["align"], s["packed"]
    flat = ids.reshape(-1)
    starts, source, position = [0], np.full(m, -1), np.full(flat.shape, -1)
    for e in range(case["experts"]):
        mine = np.nonzero(flat == e)[0]
        source[starts[-1] : starts[-1] + mine.size] = mine
        position[mine] = starts[-1] + np.arange(mine.size)
        starts.append(starts[-1] + -(-mine.size // align) * align)
    row = torch.from_numpy(np.nonzero(source >= 0)[0]).to(DEVICE)
    assignment = torch.from_numpy(source[source >= 0]).to(DEVICE)
    token = assignment // k
    w = s["weights"].double().reshape(-1)[assignment][:, None]
    x = s["x"].double()
    packed = torch.zeros((m, x.shape[1]), dtype=torch.float64, device=DEVICE)
    packed[row] = x[token]
    back = lambda v: torch.zeros_like(x).index_add_(0, token, v)  # noqa: E731
    y = s["y"].double()[row]
    i64 = lambda v: torch.from_numpy(np.asarray(v, dtype=np.int64))  # noqa: E731
    got = i64(starts), i64(source), i64(position.reshape(ids.shape)), packed, back(y * w)
    if case["kind"] == "experts":
        return got
    g = s["g_out"].double()
    g_y, g_w = torch.zeros_like(packed), torch.zeros(flat.shape, dtype=torch.float64, device=DEVICE)
    g_y[row] = g[token] * w
    g_w[assignment] = (y * g[token]).sum(1)
    return got + (back(s["g_packed"].double()[row]), g_y, g_w.reshape(ids.shape))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("score", "policy"):
        return _exact_logits(case, s)
    if case["kind"] in ("experts", "route"):
        return _exact_experts(case, s)
    live = torch.nonzero(s["tokens"] >= 0)[:, 0]
    out = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device=DEVICE)
    out[live] = s["table"].double()[s["tokens"][live]] * case["scale"]
    if case["kind"] == "embed":
        return out
    grad = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEVICE)
    order = torch.argsort(s["tokens"][live])
    token, count = torch.unique_consecutive(s["tokens"][live][order], return_counts=True)
    last = torch.cumsum(s["grad"][live[order]].double(), 0)[count.cumsum(0) - 1]  # sums of runs, as differences of running sums
    last[1:] -= last[:-1].clone()
    grad[token] = last * case["scale"]
    return out, grad
