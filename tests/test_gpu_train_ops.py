"""The scoring and training operators against their plain forms in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32, half a step of bf16 2^-9 of a value's power of two (2^-8 relative at most).
Exponents are (x - m) c2 with three roundings, so an exponential of distance D = (m - x) / T in natural units is off by 3 u D
relative, plus 4 u of the hardware's exp2 and its neighbours; where it weighs anything in a sum, D exp(-D) < 1 of the whole.  Sums of V
terms run through chains of V / 1024 + 32 additions or fewer.
"""
import numpy as np
import pytest

from gpu_common import have_gpu
from oracle import train_rows as tr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not have_gpu():
        pytest.skip("no GPU")


def ap():
    import paper_2509_18521_amd
    return paper_2509_18521_amd


def types():
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def half(t):
    """Largest rounding to a type, relative to the value."""
    return 2.0 ** -8 if t == "bf16" else U


def place(a, t, pad=0, off=0):
    """A GPU tensor of the values (rounded to the type) inside a wider one, `off` elements from a 16-byte border, rows `pad` elements longer."""
    import torch
    a = torch.as_tensor(np.asarray(a, dtype=np.float32)).to(types()[t])
    n, m = a.shape
    flat = torch.full((n * (m + pad) + off + 8,), 7.0, dtype=a.dtype, device="cuda")
    x = flat[off:off + n * (m + pad)].view(n, m + pad)[:, :m]
    x.copy_(a)
    return x


def host(x):
    return x.detach().double().cpu().numpy() if x.is_floating_point() else x.cpu().numpy()


def index(a, bits):
    import torch
    return torch.as_tensor(np.asarray(a), dtype=torch.int32 if bits == 32 else torch.int64).cuda()


def f32(a):
    import torch
    return torch.as_tensor(np.asarray(a, dtype=np.float32)).cuda()


def near(got, want, tol, what=""):
    got, want, tol = np.broadcast_arrays(np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64), np.asarray(tol, dtype=np.float64))[:3]
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    want = np.where(np.isnan(want) | (np.abs(want) < 2.0 ** 128 * (1 - 2.0 ** -25)), want, np.copysign(np.inf, want))     # (what fp32 rounds to infinity)
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    there = np.isfinite(want)
    off = np.abs(got[there] - want[there]) - tol[there]
    assert off.size == 0 or np.max(off) <= 0, (what, float(np.max(off)), got[there][np.argmax(off)], want[there][np.argmax(off)])


# --- log-probabilities ------------------------------------------------------------------------------------------------------


def hard_logits(rng, n, vocab, t):
    """Ordinary rows, and rows where something can go wrong."""
    x = (2.5 * rng.standard_normal((n, vocab))).astype(np.float32)
    low = -3.3895313892515355e38 if t == "bf16" else np.finfo(np.float32).min
    for r in range(n):
        kind = r % 16
        some = rng.random(vocab) < 0.7
        if kind == 1:
            x[r] = 0.0                                       # nothing but ties
        elif kind == 2:
            x[r, some] = -np.inf
            x[r, rng.integers(vocab)] = 0.5
        elif kind == 3:
            x[r] = low                                       # masks of the type's lowest value, the whole row
        elif kind == 4:
            x[r, some] = low
        elif kind == 5:
            x[r] = -np.inf
        elif kind == 6:
            x[r, rng.integers(vocab)] = np.nan
        elif kind == 7:
            x[r, rng.integers(vocab)] = np.inf
        elif kind == 8:
            x[r] += 3e4                                      # far from zero
        elif kind == 9:
            x[r] = np.sort(x[r])                             # each one a new maximum
        elif kind == 10:
            x[r, rng.integers(vocab)] = 60.0                 # certain
        elif kind == 11:
            x[r] = -np.inf
            x[r, -1] = -5.0                                  # a single one, the last
        elif kind == 12:
            x[r] = np.where(some, 0.0, -0.0)                 # both zeros are equal
        elif kind == 13:
            x[r, : vocab // 2] = 3e38
            x[r, vocab // 2:] = low
        elif kind == 14:
            x[r] = np.round(x[r])                            # many ties
        elif kind == 15:
            x[r] = np.sort(x[r])[::-1]
    return x


def check_logprobs(x, tokens, t, *, temperature=1.0, top=0, bits=64, pad=0, off=0):
    """The operator on these logits against the plain form; returns (logits on the GPU, its result, the logits in 64 bits)."""
    logits = place(x, t, pad, off)
    x = host(logits)
    got = ap().april_logprobs(logits, index(tokens, bits), temperature=temperature, entropy=True, lse=True, top=top)
    lp, ent, lse, best, ids = tr.logprobs(x, tokens, temperature, top)
    vocab = x.shape[1]
    m = np.max(np.where(np.isfinite(x), x, -np.inf), axis=1)
    with np.errstate(invalid="ignore", over="ignore"):
        dist = np.array([(m[r] - x[r, k]) / temperature if 0 <= k < vocab else 0.0 for r, k in enumerate(tokens)])
        base = U * (2 * np.log(vocab) + vocab / 1024 + 48)
        near(host(got.logprob), lp, base + 4 * U * np.abs(dist), "logprob")
        near(host(got.entropy), ent, base * (2 + np.log(vocab)), "entropy")
        near(host(got.lse), lse, base + 4 * U * np.abs(lse), "lse")
        if top:
            assert np.array_equal(host(got.top_ids), ids)
            near(host(got.top_logprobs), best, base + 4 * U * np.abs(best), "top")
    return logits, got, x


SIZES = [(1, 1), (3, 2), (17, 7), (16, 64), (33, 300), (16, 512), (17, 1000), (16, 4099), (5, 8192), (20, 32003), (16, 151936)]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", SIZES)
def test_logprobs(n, vocab, t):
    rng = np.random.default_rng([n, vocab, t == "f32"])
    tokens = rng.integers(0, vocab, size=n)
    if n > 16:
        tokens[16] = -1
    if n > 2:
        tokens[0] = vocab
    for i, top in enumerate({0, min(5, vocab), min(64, vocab)}):
        check_logprobs(hard_logits(rng, n, vocab, t), tokens, t, temperature=(1.0, 0.6, 1.3)[i], top=top, bits=(32, 64)[i % 2])


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,pad,off", [(5, 777, 3, 1), (9, 1024, 0, 3), (16, 5000, 8, 5), (3, 6, 0, 7), (40, 30, 1, 0), (2, 40001, 15, 4)])
def test_logprobs_of_rows_at_any_address(n, vocab, pad, off, t):
    rng = np.random.default_rng([n, vocab, pad, off])
    check_logprobs(hard_logits(rng, n, vocab, t), rng.integers(0, vocab, size=n), t, top=min(20, vocab), pad=pad, off=off)


@pytest.mark.parametrize("n", [1, 2, 31, 100, 255, 256, 600])
def test_logprobs_of_few_and_many_rows(n):
    """However the rows are shared out between workgroups; the same call twice has the same bits."""
    rng = np.random.default_rng(n)
    x = hard_logits(rng, n, 9000, "bf16")
    tokens = rng.integers(0, 9000, size=n)
    logits, got, _ = check_logprobs(x, tokens, "bf16", top=20)
    again = ap().april_logprobs(logits, index(tokens, 32), entropy=True, lse=True, top=20)
    for a, b in zip(got, again):
        assert np.array_equal(host(a), host(b), equal_nan=True)


def test_logprobs_of_all_kinds_of_ties():
    """Lists of candidates longer than any buffer: equal logits, blocks of equal ones, long runs above the rest at any stride."""
    rng = np.random.default_rng(8)
    vocab = 50000
    rows = [np.zeros(vocab), np.where(np.arange(vocab) % 8 == 3, 1.0, 0.0), np.where(np.arange(vocab) > 45000, 2.0, 1.0), np.where(np.arange(vocab) < 3000, rng.random(vocab) + 5, 0.0),
            np.where(np.arange(vocab) % 1024 == 17, rng.random(vocab) + 5, 0.0), np.where(np.arange(vocab) % 4096 < 8, rng.random(vocab) + 5, rng.random(vocab)),
            np.where(np.arange(vocab) % 8192 < 512, rng.random(vocab) + 5, 0.0), np.where(np.arange(vocab) % 16 == 0, -1.0, -np.inf), np.full(vocab, -np.inf),
            np.arange(vocab) / 64.0, -np.arange(vocab) / 64.0, rng.integers(0, 3, size=vocab).astype(float)]
    rows[8][[40000, 7, 49999]] = (1.0, 2.0, 1.0)
    x = np.array(rows)
    for t in ("bf16", "f32"):
        for top in (1, 3, 64):
            check_logprobs(x, rng.integers(0, vocab, size=len(rows)), t, top=top)
            check_logprobs(np.tile(x, (30, 1)), rng.integers(0, vocab, size=30 * len(rows)), t, top=top) if top == 64 else None


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,pad,off", [(1, 0, 0), (5, 3, 1), (64, 0, 0), (300, 0, 2), (513, 6, 5), (1001, 0, 0), (5000, 1, 3), (7999, 0, 0), (16000, 0, 0), (16384, 8, 0)])
def test_logprobs_of_many_short_rows(vocab, pad, off, t):
    """Thousands of rows, among them those whose ties and blocks of large values fill any list: copies of a row at like addresses have the same bits, and those of 48 rows are checked."""
    import torch
    rng = np.random.default_rng([vocab, pad, off])
    x = hard_logits(rng, 48, vocab, t)
    i = np.arange(vocab)
    x[16], x[17], x[18] = i % 3, np.where(i % 64 < 8, 5.0 + i / 64.0, 0.0), np.where(i % 512 < 32, 7.0, rng.standard_normal(vocab))
    x[19], x[20] = np.where(i % 16 == 0, -1.0, -np.inf), np.where(i < 1000, 3.0, 1.0)
    tokens = rng.integers(0, vocab, size=48)
    tokens[[5, 30]] = -1, vocab
    n = 2500
    of = rng.integers(0, 48, size=n)
    of[:48] = np.arange(48)
    for top in sorted({0, 1, min(20, vocab), min(32, vocab), min(33, vocab)}):
        _, few, _ = check_logprobs(x, tokens, t, top=top)
        logits = place(x[of], t, pad, off)
        got = ap().april_logprobs(logits, index(tokens[of], 64), entropy=True, lse=True, top=top)
        lp, ent, lse, best, ids = tr.logprobs(host(logits[:48]), tokens, 1.0, top)
        near(host(got.logprob)[:48], host(few.logprob), 2e-6 * (1 + np.abs(np.nan_to_num(host(few.logprob), posinf=0, neginf=0))), "logprob")
        near(host(got.entropy)[:48], ent, U * (2 * np.log(vocab) + vocab / 64 + 48) * (2 + np.log(vocab)), "entropy")
        assert not top or np.array_equal(host(got.top_ids)[:48], ids)
        assert not top or torch.equal(got.top_ids, got.top_ids[:48][torch.as_tensor(of).cuda()])
        first, per = {}, 8 if t == "bf16" else 4             # (a row's sums go by its place to a 16-byte border)
        same = torch.as_tensor([first.setdefault((of[r], (off + r * (vocab + pad)) % per), r) for r in range(n)]).cuda()
        for v in got:
            if v is not None:
                assert torch.equal(v.nan_to_num(nan=123.0), v[same].nan_to_num(nan=123.0))


def check_grad(n, vocab, t, temperature, parts, *, pad=0, off=0, in_place=False, seed=0):
    import torch
    rng = np.random.default_rng([n, vocab, seed])
    x = hard_logits(rng, n, vocab, t)
    tokens = rng.integers(0, vocab, size=n)
    if n > 3:
        tokens[3] = -1
    if n > 8:
        tokens[8] = vocab + 5
    logits, made, x = check_logprobs(x, tokens, t, temperature=temperature, pad=pad, off=off)
    g, h, z = (rng.standard_normal(n).astype(np.float32) if c in parts else None for c in "ghz")
    want, size = tr.logprobs_grad(x, tokens, temperature, *(None if v is None else v.astype(np.float64) for v in (g, h, z)))
    out = logits if in_place else None if pad == off == 0 else place(np.zeros((n, vocab)), t, pad + 1, off + 1)
    around = None if in_place or out is None else out.as_strided((n, vocab + pad + 1), out.stride()).clone()
    got = ap().april_logprobs_grad(logits, index(tokens, 64), made, grad_logprob=None if g is None else f32(g), grad_entropy=None if h is None else f32(h),
                                   grad_lse=None if z is None else f32(z), temperature=temperature, out=out)
    assert out is None or got is out
    finite = np.isfinite(x).any(axis=1) & ~np.isnan(x).any(axis=1) & ~(x == np.inf).any(axis=1)
    for r in np.nonzero(~finite & (tokens >= 0))[0]:
        assert np.isnan(host(got)[r]).all(), r
    keep = finite | (tokens < 0)
    with np.errstate(invalid="ignore", over="ignore"):
        m = np.max(np.where(np.isfinite(x), x, -np.inf), axis=1, keepdims=True)
        dist = np.minimum(np.abs(np.nan_to_num(m - x, nan=0.0, posinf=0.0, neginf=0.0)) / temperature, 200.0)
    # each term: an exponential of that distance, the forward's log of the sum and entropy, a handful of products
    rel = U * (6 * dist + 4 * np.log(vocab) + vocab / 1024 + 64) * (3 if h is not None else 1)
    tol = size * rel + half(t) * np.abs(want) + 1e-37 * (1 + np.nan_to_num(size)) + (2.0 ** -133 if t == "bf16" else 2.0 ** -149)
    near(host(got)[keep], want[keep], tol[keep], "gradient")
    if around is not None:
        around[:, :vocab] = 0
        left = out.as_strided((n, vocab + pad + 1), out.stride())[: n - 1].clone()
        left[:, :vocab] = 0
        assert torch.equal(left.nan_to_num(), around[: n - 1].nan_to_num())              # nothing between the rows


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", SIZES)
def test_logprobs_grad(n, vocab, t):
    check_grad(n, vocab, t, 1.0, "ghz")
    check_grad(n, vocab, t, 0.7, "g", in_place=True, seed=1)


@pytest.mark.parametrize("parts", ["", "h", "z", "gh", "hz"])
def test_logprobs_grad_parts(parts):
    check_grad(37, 2000, "bf16", 1.4, parts)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,pad,off", [(5, 777, 3, 1), (9, 1024, 0, 3), (17, 5000, 8, 5), (3, 6, 0, 7), (2, 40001, 15, 4)])
def test_logprobs_grad_at_any_address(n, vocab, pad, off, t):
    check_grad(n, vocab, t, 1.0, "gh", pad=pad, off=off)
    check_grad(n, vocab, t, 1.0, "gh", pad=pad, off=off, in_place=True)


def test_logprobs_autograd_is_the_gradient():
    """Through autograd, with a gradient that is one expanded number, through a row that is repeated, and against differences."""
    import torch
    rng = np.random.default_rng(4)
    x = rng.standard_normal((6, 50)).astype(np.float32)
    tokens = index([3, 49, -1, 0, 7, 7], 64)
    leaf = torch.as_tensor(x).cuda().requires_grad_()
    got = ap().april_logprobs(leaf, tokens, temperature=0.8, entropy=True, lse=True, top=4)
    assert not got.top_logprobs.requires_grad and not got.top_ids.requires_grad and not got.norm.requires_grad
    (got.logprob.sum() + 0.3 * got.entropy.mean() - got.lse.square().sum()).backward()
    lse = tr.logprobs(x, host(tokens), 0.8)[2]
    want, size = tr.logprobs_grad(x, host(tokens), 0.8, np.ones(6), np.full(6, 0.05), -2 * lse)
    near(host(leaf.grad), want, size * U * 200 + U)
    base = torch.as_tensor(x[:1]).cuda().requires_grad_()
    one = ap().april_logprobs(base.expand(6, 50), tokens)
    one.logprob.sum().backward()
    w, s = tr.logprobs_grad(np.repeat(x[:1], 6, 0), host(tokens), 1.0, np.ones(6))
    near(host(base.grad), w.sum(0, keepdims=True), s.sum(0, keepdims=True) * U * 200 + U)

    def loss(v):
        lp, ent, _, _, _ = tr.logprobs(v, host(tokens), 0.8)
        return lp.sum() + 0.3 * ent.mean()
    d = rng.standard_normal(x.shape)
    leaf.grad = None
    got = ap().april_logprobs(leaf, tokens, temperature=0.8, entropy=True)
    (got.logprob.sum() + 0.3 * got.entropy.mean()).backward()
    along = (loss(x + 1e-5 * d) - loss(x - 1e-5 * d)) / 2e-5
    assert abs(np.sum(host(leaf.grad) * d) - along) < 1e-4
    with torch.no_grad():
        assert not ap().april_logprobs(leaf, tokens).logprob.requires_grad
    with pytest.raises(RuntimeError):                        # what it was computed from is gone
        got = ap().april_logprobs(leaf * 1.0, tokens)
        y = leaf * 1.0
        got = ap().april_logprobs(y, tokens)
        y.zero_()
        got.logprob.sum().backward()


# --- embedding ---------------------------------------------------------------------------------------------------------------


def tokens_of(rng, n, vocab, kind):
    if kind == "one":
        t = np.full(n, vocab // 2)
    elif kind == "skewed":
        t = np.minimum(np.exp(rng.random(n) * np.log(vocab)).astype(np.int64), vocab) - 1
    elif kind == "none":
        t = np.full(n, -1)
    elif kind == "sorted":
        t = np.sort(rng.integers(0, vocab, size=n))
    else:
        t = rng.integers(0, vocab, size=n)
    if n > 4 and kind not in ("none", "one"):
        t[rng.integers(n)] = -1
        t[rng.integers(n)] = vocab
        t[rng.integers(n)] = -(1 << 30)
    return t


EMBED = [(1, 1, 1, "any"), (1, 151936, 8, "any"), (5, 3, 7, "any"), (64, 512, 128, "any"), (200, 9, 33, "skewed"), (1000, 100, 64, "one"), (129, 5, 16, "one"), (128, 5, 16, "one"),
         (513, 700, 1037, "skewed"), (4097, 1000, 24, "skewed"), (9000, 40000, 40, "skewed"), (5000, 511, 8, "sorted"), (5000, 512, 8, "any"), (300, 300000, 4, "any"), (77, 50, 100, "none"),
         (20000, 3, 12, "any")]


@pytest.mark.parametrize("tt,to", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,vocab,d,kind", EMBED)
def test_embed_and_its_gradient(n, vocab, d, kind, tt, to):
    import torch
    rng = np.random.default_rng([n, vocab, d])
    scale = 1.0 if d % 2 else 11.3
    pad, off = (0, 0) if n % 3 else (5, 3)
    table = place(rng.standard_normal((vocab, d)), tt, pad, off)
    tokens = tokens_of(rng, n, vocab, kind)
    idx = index(tokens, 32 if n % 2 else 64)
    s = float(np.float32(scale))
    got = ap().april_embed(table, idx, scale=scale, dtype=types()[to])
    assert got.dtype is types()[to]
    want = tr.embed(host(table), tokens, s)
    near(host(got), want, (U + half(to)) * np.abs(want))
    grad = place(rng.standard_normal((n, d)), to, pad, off)
    want, size, rows = tr.embed_grad(host(grad), tokens, vocab, s)
    depth = np.minimum(rows, 128) + rows // 128 + 2
    tol = depth[:, None] * U * size + half(tt) * np.abs(want)
    got = ap().april_embed_grad(grad, idx, vocab, scale=scale, dtype=types()[tt])
    near(host(got), want, tol)
    assert torch.equal(got, ap().april_embed_grad(grad, idx, vocab, scale=scale, dtype=types()[tt]))
    start = place(rng.standard_normal((vocab, d)), tt, pad, off)
    before = start.clone()
    want, size, _ = tr.embed_grad(host(grad), tokens, vocab, s, host(before))
    again = ap().april_embed_grad(grad, idx, vocab, scale=scale, out=start, accumulate=True)
    assert again is start
    near(host(start), want, (depth[:, None] + 1) * U * size + half(tt) * np.abs(want))
    assert torch.equal(start[torch.as_tensor(rows == 0).cuda()], before[torch.as_tensor(rows == 0).cuda()])
    if pad:
        whole = start.as_strided((vocab, d + pad), start.stride())[: vocab - 1, d:]
        assert bool((whole == 7.0).all())                    # nothing between the rows


def test_embed_autograd():
    import torch
    rng = np.random.default_rng(6)
    table = torch.as_tensor(rng.standard_normal((30, 9)), dtype=torch.float32).cuda().requires_grad_()
    tokens = index([3, 3, -1, 29, 0, 3], 64)
    out = ap().april_embed(table, tokens, scale=3.0)
    out.sum().backward()                                     # (a gradient that is one expanded number)
    want, size, _ = tr.embed_grad(np.ones((6, 9)), host(tokens), 30, 3.0)
    near(host(table.grad), want, 4 * U * size)
    table.grad = None
    g = torch.as_tensor(rng.standard_normal((9, 6)), dtype=torch.float32).cuda().T
    ap().april_embed(table, tokens).backward(g)              # columns adjacent
    want, size, _ = tr.embed_grad(host(g), host(tokens), 30)
    near(host(table.grad), want, 4 * U * size)
    with pytest.raises(ap().AprilError, match="out|table"):
        ap().april_embed(table, tokens, out=torch.empty((6, 9), device="cuda"))


def test_embed_grad_of_no_rows():
    import torch
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    got = ap().april_embed_grad(torch.empty((0, 12), device="cuda"), none, 40)
    assert got.shape == (40, 12) and not bool(got.any())
    start = torch.ones((40, 12), device="cuda")
    ap().april_embed_grad(torch.empty((0, 12), device="cuda"), none, 40, out=start, accumulate=True)
    assert bool((start == 1).all())
    assert ap().april_embed(start, none).shape == (0, 12)
    assert ap().april_logprobs(torch.empty((0, 9), device="cuda"), none, top=3).top_ids.shape == (0, 3)


# --- experts -----------------------------------------------------------------------------------------------------------------

EXPERTS = [(1, 1, 1, 1, 1), (1, 8, 128, 64, 64), (3, 2, 5, 7, 4), (70, 4, 16, 128, 16), (384, 8, 128, 24, 64), (500, 3, 1, 10, 1), (513, 8, 64, 33, 128), (1500, 6, 511, 9, 8), (4000, 2, 7, 16, 1),
           (9, 64, 100, 12, 3), (300, 10, 200, 520, 1)]


def expert_ids(rng, n, k, e, out_of_range):
    ids = rng.integers(0, e, size=(n, k))
    if n > 10:
        ids[: n // 2] = np.minimum(rng.integers(0, e, size=(n // 2, k)), rng.integers(0, e, size=(n // 2, k)))   # uneven shares
    if out_of_range:
        ids[rng.random((n, k)) < 0.2] = -1
        ids[rng.random((n, k)) < 0.1] = e
        ids[0] = -5
    return ids


@pytest.mark.parametrize("lost", [False, True])
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("n,k,e,d,align", EXPERTS)
def test_experts(n, k, e, d, align, t, lost):
    import torch
    rng = np.random.default_rng([n, k, e, d])
    ids = expert_ids(rng, n, k, e, lost)
    rows = ap().april_expert_sort(index(ids, 64 if lost else 32), e, align=align)
    starts, source, position = tr.expert_sort(ids, e, align)
    assert np.array_equal(host(rows.starts), starts) and np.array_equal(host(rows.source), source) and np.array_equal(host(rows.position), position)
    m = len(source)
    pad, off = (0, 0) if n % 2 else (3, 5)
    x = place(rng.standard_normal((n, d)), t, pad, off)
    packed = ap().april_expert_gather(x, rows)
    assert np.array_equal(host(packed), tr.expert_gather(host(x), source, k))
    y = rng.standard_normal((m, d))
    y[source < 0] = np.nan                                   # what lies between is not read
    y = place(y, t, pad, off)
    w = rng.random((n, k)).astype(np.float32)
    for weights in (None, w):
        got = ap().april_expert_combine(y, rows, None if weights is None else f32(weights))
        want, size = tr.expert_combine(host(y), position, weights)
        near(host(got), want, (k + 1) * U * size + half(t) * np.abs(want))
        g = place(rng.standard_normal((n, d)), t, pad, off)
        g_y, g_w = ap().april_expert_combine_grad(g, y, rows, None if weights is None else f32(weights))
        want_y, want_w, size_w = tr.expert_combine_grad(host(g), host(y), source, position, weights)
        near(host(g_y), want_y, (U + half(t)) * np.abs(want_y))
        near(host(g_w), want_w, (d + 8) * U * size_w)
        only, none = ap().april_expert_combine_grad(g, y, rows, None if weights is None else f32(weights), of_weights=False)
        assert none is None and torch.equal(only, g_y)
        none, only = ap().april_expert_combine_grad(g, y, rows, None if weights is None else f32(weights), of_packed=False)
        assert none is None and torch.equal(only, g_w)


def test_experts_of_no_rows():
    import torch
    rows = ap().april_expert_sort(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 6, align=16)
    assert host(rows.starts).tolist() == [0] * 7 and rows.source.shape == (0,) and rows.position.shape == (0, 4)
    packed = ap().april_expert_gather(torch.empty((0, 32), device="cuda"), rows)
    assert packed.shape == (0, 32) and ap().april_expert_combine(packed, rows).shape == (0, 32)
    of_packed, of_weights = ap().april_expert_combine_grad(packed, packed, rows)
    assert of_packed.shape == (0, 32) and of_weights.shape == (0, 4)


def test_experts_of_entries_outside_their_arrays():
    """A source or position that is none of the arrays' counts as -1 (and nothing outside is read)."""
    import torch
    rng = np.random.default_rng(2)
    x = place(rng.standard_normal((4, 16)), "f32")
    rows = ap().ExpertRows(index([0, 8], 32), index([0, 900, -7, 3, 2 ** 31 - 1, 7, 1, -1], 32), index([[0, 6], [-9, 3], [8, 2 ** 31 - 1], [77, 5]], 32))
    source = np.array([0, -1, -1, 3, -1, 7, 1, -1])
    assert np.array_equal(host(ap().april_expert_gather(x, rows)), tr.expert_gather(host(x), source, 2))
    y = place(rng.standard_normal((8, 16)), "f32")
    position = np.array([[0, 6], [-1, 3], [-1, -1], [-1, 5]])
    want, size = tr.expert_combine(host(y), position)
    near(host(ap().april_expert_combine(y, rows)), want, 3 * U * size)
    g_y, g_w = ap().april_expert_combine_grad(x, y, rows)
    want_y, want_w, size_w = tr.expert_combine_grad(host(x), host(y), source, position)
    near(host(g_y), want_y, U * np.abs(want_y))
    near(host(g_w), want_w, 24 * U * size_w)
    assert torch.equal(g_y[4], torch.zeros(16, device="cuda"))


def test_experts_autograd():
    import torch
    rng = np.random.default_rng(9)
    n, k, e, d = 40, 3, 7, 20
    ids = expert_ids(rng, n, k, e, True)
    rows = ap().april_expert_sort(index(ids, 64), e, align=4)
    _, source, position = tr.expert_sort(ids, e, 4)
    x, w = f32(rng.standard_normal((n, d))).requires_grad_(), f32(rng.random((n, k))).requires_grad_()
    packed = ap().april_expert_gather(x, rows)
    out = ap().april_expert_combine(packed * 2.0, rows, w)
    out.sum().backward()
    g_y, g_w, size_w = tr.expert_combine_grad(np.ones((n, d)), 2 * host(packed), source, position, host(w))
    g_x, size_x = tr.expert_combine(2 * g_y, position)
    near(host(w.grad), g_w, (d + 8) * U * size_w)
    near(host(x.grad), g_x, 8 * U * size_x)
    assert w.grad is not None
    x.grad = None
    ap().april_expert_combine(ap().april_expert_gather(x, rows), rows).sum().backward()
    assert x.grad is not None


# --- what is not read, and what is large --------------------------------------------------------------------------------------


def test_padding_is_not_read():
    """NaN in rows of padding, in weights of assignments that are left out, in packed rows of none."""
    import torch
    rng = np.random.default_rng(30)
    n, vocab, d, k, e = 60, 1000, 40, 3, 8
    tokens = rng.integers(0, vocab, size=n)
    tokens[::3] = -1
    off = torch.as_tensor(tokens < 0).cuda()
    idx = index(tokens, 64)
    logits = place(rng.standard_normal((n, vocab)), "f32")
    want = ap().april_logprobs(logits, idx, entropy=True, top=4)
    g = f32(rng.standard_normal(n))
    want_grad = ap().april_logprobs_grad(logits, idx, want, grad_logprob=g, grad_entropy=g)
    logits[off] = float("nan")
    got = ap().april_logprobs(logits, idx, entropy=True, top=4)
    g[off] = float("nan")
    for a, b in zip(got, want):
        assert a is b is None or torch.equal(a, b)
    assert torch.equal(ap().april_logprobs_grad(logits, idx, got, grad_logprob=g, grad_entropy=g), want_grad) and not bool(want_grad[off].any())
    grad = place(rng.standard_normal((n, d)), "bf16")
    want = ap().april_embed_grad(grad, idx, vocab)
    grad[off] = float("nan")
    assert torch.equal(ap().april_embed_grad(grad, idx, vocab), want) and not bool(want.isnan().any())
    ids = expert_ids(rng, n, k, e, True)
    rows = ap().april_expert_sort(index(ids, 64), e, align=16)
    w = f32(rng.random((n, k)))
    y = place(rng.standard_normal((rows.source.shape[0], d)), "f32")
    want = [ap().april_expert_combine(y, rows, w), *ap().april_expert_combine_grad(f32(np.ones((n, d))), y, rows, w)]
    w[rows.position < 0] = float("nan")
    y[rows.source < 0] = float("nan")
    got = [ap().april_expert_combine(y, rows, w), *ap().april_expert_combine_grad(f32(np.ones((n, d))), y, rows, w)]
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_logprobs_of_more_elements_than_31_bits_count():
    import torch
    n, vocab = 14200, 151936
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.empty((n, vocab), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    tokens = torch.randint(vocab, (n,), generator=gen, device="cuda")
    got = ap().april_logprobs(logits, tokens, entropy=True, top=3)
    g = torch.randn(n, generator=gen, device="cuda")
    grad = ap().april_logprobs_grad(logits, tokens, got, grad_logprob=g, grad_entropy=g)
    for r in (0, 14133, 14134, 14140, n - 1):                # (2^31 elements end in row 14134)
        x, t = host(logits[r:r + 1]), host(tokens[r:r + 1])
        lp, ent, _, best, ids = tr.logprobs(x, t, 1.0, 3)
        near(host(got.logprob[r:r + 1]), lp, U * 300)
        near(host(got.entropy[r:r + 1]), ent, U * 3000)
        assert np.array_equal(host(got.top_ids[r:r + 1]), ids)
        want, size = tr.logprobs_grad(x, t, 1.0, host(g[r:r + 1]), host(g[r:r + 1]))
        near(host(grad[r:r + 1]), want, size * U * 1000 + half("bf16") * np.abs(want) + 2.0 ** -133)
    ap().april_logprobs_grad(logits, tokens, got, grad_logprob=g, grad_entropy=g, out=logits)
    assert torch.equal(logits, grad)


def test_rows_of_more_elements_than_31_bits_count():
    import torch
    vocab, d, n = 270000, 8192, 40
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    tokens = torch.randint(vocab, (n,), generator=gen, device="cuda")
    tokens[:4] = torch.tensor([0, vocab - 1, 262143, 262144])
    out = ap().april_embed(table, tokens)
    assert torch.equal(out, table[tokens])
    grad = ap().april_embed_grad(out, tokens, vocab)
    want, _, rows = tr.embed_grad(host(out), host(tokens), vocab)
    there = np.nonzero(rows)[0]
    near(host(grad[torch.as_tensor(there).cuda()]), want[there], half("bf16") * np.abs(want[there]))
    assert int((grad != 0).any(1).sum()) == len(there)
    del grad
    # as packed rows: the token's row at its own place
    rows = ap().ExpertRows(torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((vocab,), -1, dtype=torch.int32, device="cuda"), tokens.int()[:, None].contiguous())
    rows.source[tokens] = torch.arange(n, dtype=torch.int32, device="cuda")
    assert torch.equal(ap().april_expert_combine(table, rows), out)
    packed = ap().april_expert_gather(out, rows)
    assert torch.equal(packed[tokens], out) and int((packed != 0).any(1).sum()) == len(there)
    g_packed, g_weights = ap().april_expert_combine_grad(out, table, rows)
    assert torch.equal(g_packed, packed)
    near(host(g_weights[:, 0]), (host(out) ** 2).sum(1), d * U * (host(out) ** 2).sum(1))


@pytest.mark.parametrize("d", [8192, 8191])
def test_rows_past_the_last_cache(d):
    """Sizes whose accesses are streamed, whole vectors and rows with a tail; whole numbers, whose sums are exact."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(d)
    whole = lambda *s: torch.randint(-8, 9, s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    n, vocab, k, e = 9000, 9500, 8, 16
    table, g, tokens = whole(vocab, d), whole(n, d), torch.randint(-5, vocab, (n,), generator=gen, device="cuda")
    tokens[::9] = 123
    keep = tokens >= 0
    assert torch.equal(ap().april_embed(table, tokens), torch.where(keep[:, None], table[tokens.clamp(min=0)], 0))
    want = torch.zeros((vocab, d), device="cuda").index_add_(0, tokens[keep], g[keep].float()).bfloat16()
    assert torch.equal(ap().april_embed_grad(g, tokens, vocab), want)
    start = table.clone()
    ap().april_embed_grad(g, tokens, vocab, out=start, accumulate=True)
    assert torch.equal(start, (table.float() + torch.zeros((vocab, d), device="cuda").index_add_(0, tokens[keep], g[keep].float())).bfloat16())
    del table, start, want
    x = g[:1200]
    ids = torch.randint(-1, e, (1200, k), generator=gen, device="cuda")
    rows = ap().april_expert_sort(ids, e, align=64)
    there, token = rows.source >= 0, rows.source.clamp(min=0).long() // k
    packed = ap().april_expert_gather(x, rows)
    assert torch.equal(packed, torch.where(there[:, None], x[token], 0))
    position = rows.position.long()
    want = (x.float() * (position >= 0).sum(1)[:, None]).bfloat16()
    assert torch.equal(ap().april_expert_combine(packed, rows), want)
    w = torch.randint(1, 4, (1200, k), generator=gen, device="cuda").float()
    g_packed, g_weights = ap().april_expert_combine_grad(x, packed, rows, w)
    assert torch.equal(g_packed, torch.where(there[:, None], x[token].float() * w.reshape(-1)[rows.source.clamp(min=0).long()][:, None], 0).bfloat16())
    assert torch.equal(g_weights, torch.where(position >= 0, x.float().square().sum(1)[:, None], 0))


def test_sorts_of_many_tiles():
    """More tiles than a workgroup adds up by itself."""
    import torch
    n, k, e = 150001, 8, 300
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(-3, e + 3, (n, k), generator=gen, device="cuda")
    rows = ap().april_expert_sort(ids, e, align=8)
    flat = ids.reshape(-1).cpu().numpy()
    there = (flat >= 0) & (flat < e)
    count = np.bincount(flat[there], minlength=e)
    starts = np.concatenate(([0], np.cumsum((count + 7) // 8 * 8)))
    assert np.array_equal(host(rows.starts), starts)
    order = np.argsort(np.where(there, flat, e), kind="stable")[: there.sum()]
    place_of = starts[flat[order]] + np.arange(len(order)) - np.concatenate(([0], np.cumsum(count)))[flat[order]]
    source, position = np.full(rows.source.shape[0], -1), np.full(n * k, -1)
    source[place_of], position[order] = order, place_of
    assert np.array_equal(host(rows.source), source) and np.array_equal(host(rows.position).reshape(-1), position)
    n, vocab, d = 1100003, 5003, 5
    tokens = torch.randint(-20, vocab + 20, (n,), generator=gen, device="cuda")
    tokens[torch.rand(n, generator=gen, device="cuda") < 0.4] = 77
    g = torch.randint(-8, 9, (n, d), generator=gen, device="cuda").float()     # (sums of whole numbers are exact)
    got = ap().april_embed_grad(g, tokens, vocab)
    want = torch.zeros((vocab, d), dtype=torch.float64)
    keep = (tokens >= 0) & (tokens < vocab)
    want.index_add_(0, tokens[keep].cpu(), g[keep].double().cpu())
    assert torch.equal(got.double().cpu(), want)


# --- together ----------------------------------------------------------------------------------------------------------------


def policy_step(p, tokens, targets, a, ent_weight, k, ops):
    """Loss of a small routed policy on rollouts: embedding, a layer of experts with its router, head, policy gradient with an entropy bonus."""
    import torch
    emb, router, experts, head = p
    x = ops.embed(emb, tokens)
    w, ids = torch.topk(torch.softmax(x @ router.T, 1), k)
    w = w / w.sum(1, keepdim=True)
    x = x + ops.experts(x, ids, w, experts)
    lp, ent = ops.logprobs(x @ head.T, targets)
    return -(a * lp).sum() - ent_weight * ent.sum()


class Plain:
    @staticmethod
    def embed(table, tokens):
        return table[tokens.clamp(min=0)] * (tokens >= 0)[:, None] * 1.5

    @staticmethod
    def experts(x, ids, w, experts):
        import torch
        out = 0
        for j in range(ids.shape[1]):
            out = out + w[:, j:j + 1] * torch.bmm(experts[ids[:, j]], x[:, :, None])[:, :, 0]
        return out

    @staticmethod
    def logprobs(logits, targets):
        import torch
        logp = torch.log_softmax(logits / 0.9, 1)
        keep = targets >= 0
        return logp.gather(1, targets.clamp(min=0)[:, None])[:, 0] * keep, -(logp.exp() * logp).sum(1) * keep


class Own:
    @staticmethod
    def embed(table, tokens):
        return ap().april_embed(table, tokens, scale=1.5)

    @staticmethod
    def experts(x, ids, w, experts):
        import torch
        rows = ap().april_expert_sort(ids, experts.shape[0], align=8)
        packed = ap().april_expert_gather(x, rows)
        at = rows.starts.tolist()
        made = [packed[at[i]:at[i + 1]] @ experts[i].T for i in range(experts.shape[0])] + [packed[at[-1]:] * 0]
        return ap().april_expert_combine(torch.cat(made), rows, w)

    @staticmethod
    def logprobs(logits, targets):
        got = ap().april_logprobs(logits, targets, temperature=0.9, entropy=True)
        return got.logprob, got.entropy


def test_a_training_step_of_a_routed_policy():
    """The operators one after another, forward and backward, against plain torch in 64 bits on the CPU."""
    import torch
    rng = np.random.default_rng(12)
    n, vocab, d, e, k = 150, 203, 24, 6, 2
    p = [rng.standard_normal(s) * c for s, c in (((vocab, d), 0.5), ((e, d), 1.0), ((e, d, d), 0.2), ((vocab, d), 0.5))]
    tokens, targets = tokens_of(rng, n, vocab, "skewed").clip(max=vocab - 1), rng.integers(0, vocab, size=n)
    targets[::7] = -1
    a = rng.standard_normal(n)
    grads = []
    for ops, dtype, device in ((Plain, torch.float64, "cpu"), (Own, torch.float32, "cuda")):
        q = [torch.as_tensor(v, dtype=torch.float32).to(dtype).to(device).requires_grad_() for v in p]
        ins = [torch.as_tensor(v).to(device) for v in (tokens, targets)]
        loss = policy_step(q, *ins, torch.as_tensor(a, dtype=torch.float32).to(dtype).to(device), 0.02, k, ops)
        loss.backward()
        grads.append([host(v.grad) for v in q] + [host(loss.reshape(1))])
    for i, (want, got) in enumerate(zip(*grads)):
        # sums of 150 rows x 203 tokens x 24 products in fp32, each off by a few u of its size; the tensors' own scale bounds them
        near(got, want, 3e-5 * np.max(np.abs(want)), i)


def test_logprobs_are_those_of_the_engine():
    """A rollout's tokens scored from its own logits: the engine's log-probabilities."""
    import torch
    import april_inputs as ai
    from gpu_common import make_engine, req_dicts
    shape = ai.ModelShape(2, 128, 4, 2, 64, 256, 544)
    w = ai.Workload("score", shape, 4, 20, 4, 4, 12, 2.4, 0.2, 8, 12, ai.SAMPLER_TOPK, 8, 1, 3)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, 4)
    ctx = make_engine(w, weights, debug=True, logprobs=True, temperature=0.7)
    try:
        for r in reqs:
            ap().april_debug_watch(ctx, r.request_id, 0, w.max_new)
        res = ap().april_rollout_step(ctx, req_dicts(reqs), 4, 4, w.max_new)
        for rid, toks, lps in zip(res.request_id, res.tokens, res.logprobs):
            rows = np.array([ap().april_debug_logits(ctx, rid, i, shape.vocab)[0] for i in range(len(toks))])
            got = ap().april_logprobs(f32(rows), index(toks, 32), temperature=0.7, top=1)
            dist = (np.max(rows, axis=1) - rows[np.arange(len(toks)), toks]) / 0.7
            near(host(got.logprob), lps, U * (16 * dist + 64))      # two computations of the same
            assert np.array_equal(host(got.top_ids)[:, 0], np.argmax(rows, axis=1))
    finally:
        ap().april_destroy(ctx)


def test_captured_into_a_graph():
    """Every call captured, replayed over changing inputs with eager work between, against the eager results."""
    import torch
    rng = np.random.default_rng(20)
    n, vocab, d, e, k = 300, 5003, 64, 16, 4
    logits, grad = place(rng.standard_normal((n, vocab)), "bf16"), place(rng.standard_normal((n, d)), "bf16")
    table, g = place(rng.standard_normal((vocab, d)), "bf16"), f32(rng.standard_normal(n))
    tokens, ids, w = index(tokens_of(rng, n, vocab, "skewed"), 64), index(expert_ids(rng, n, k, e, True), 32), f32(rng.random((n, k)))

    def work():
        got = ap().april_logprobs(logits, tokens, entropy=True, top=7)
        rows = ap().april_expert_sort(ids, e, align=16)
        packed = ap().april_expert_gather(grad, rows)
        out = ap().april_embed(table, tokens)
        return (got.logprob, got.entropy, got.top_logprobs, got.top_ids, ap().april_logprobs_grad(logits, tokens, got, grad_logprob=g, grad_entropy=g), *rows, packed,
                ap().april_expert_combine(packed, rows, w), *ap().april_expert_combine_grad(grad, packed, rows, w), out, ap().april_embed_grad(grad, tokens, vocab))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(4):
        logits.copy_(torch.as_tensor(rng.standard_normal((n, vocab))))
        tokens.copy_(torch.as_tensor(tokens_of(rng, n, vocab, ("skewed", "one", "any", "none")[i])))
        ids.copy_(torch.as_tensor(expert_ids(rng, n, k, e, i % 2 == 0)))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in held]
        for a, b in zip(got, work()):
            assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_captured_backward_of_fresh_leaves():
    """A whole step with autograd in a graph, the way torch asks for: warmed up on the capture's stream, no other graph of the leaves alive."""
    import torch
    rng = np.random.default_rng(21)
    n, vocab = 64, 700
    logits = place(rng.standard_normal((n, vocab)), "f32").contiguous().requires_grad_()
    tokens = index(rng.integers(0, vocab, size=n), 64)

    def step():
        logits.grad = None
        ap().april_logprobs(logits, tokens).logprob.sum().backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        with torch.no_grad():
            logits.copy_(torch.as_tensor(rng.standard_normal((n, vocab))))
        graph.replay()
        torch.cuda.synchronize()
        want, size = tr.logprobs_grad(host(logits), host(tokens), 1.0, np.ones(n))
        near(host(logits.grad), want, size * U * 200 + U * 1e-3)


def test_on_another_stream():
    import torch
    rng = np.random.default_rng(22)
    x, tokens = place(rng.standard_normal((50, 3001)), "bf16"), index(rng.integers(0, 3001, size=50), 32)
    want = ap().april_logprobs(x, tokens, entropy=True, lse=True, top=9)
    side = torch.cuda.Stream()
    y = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        y.copy_(x)                                           # (only that stream waits for this)
        got = ap().april_logprobs(y, tokens, entropy=True, lse=True, top=9)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """The same work on two streams, each call with its own workspace, side by side."""
    import torch
    rng = np.random.default_rng(23)
    n, vocab, d, e, k = 90, 60001, 96, 16, 4
    logits, grad, table = place(rng.standard_normal((n, vocab)), "f32"), place(rng.standard_normal((6000, d)), "bf16"), place(rng.standard_normal((vocab, d)), "bf16")
    tokens, many = index(rng.integers(0, vocab, size=n), 64), index(tokens_of(rng, 6000, vocab, "skewed"), 64)
    ids, w, g = index(expert_ids(rng, 6000, k, e, True), 32), f32(rng.random((6000, k))), f32(rng.standard_normal(n))

    def work():
        got = ap().april_logprobs(logits, tokens, entropy=True, top=9)
        rows = ap().april_expert_sort(ids, e, align=8)
        packed = ap().april_expert_gather(grad, rows)
        return [got.logprob, got.entropy, got.top_ids, ap().april_logprobs_grad(logits, tokens, got, grad_logprob=g, grad_entropy=g), *rows, packed, ap().april_expert_combine(packed, rows, w),
                *ap().april_expert_combine_grad(grad, packed, rows, w), ap().april_embed(table, many), ap().april_embed_grad(grad, many, vocab)]
    want = work()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = work()
    torch.cuda.synchronize()
    for side in got:
        for a, b in zip(side, want):
            assert torch.equal(a.nan_to_num(), b.nan_to_num())      # (a token beyond the table: a row of NaN)


def test_no_second_derivative():
    """A gradient of a gradient is refused by autograd, not silently zero."""
    import torch
    x = torch.randn((4, 9), device="cuda", requires_grad=True)
    t = index([1, 2, -1, 0], 64)
    (g,) = torch.autograd.grad(ap().april_logprobs(x, t).logprob.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("n", [40, 5000])
@pytest.mark.parametrize("vocab", [(1 << 27) - 1, 1 << 27, (1 << 27) + 77])
def test_embed_grad_of_the_largest_tables(vocab, n):
    """Tokens of 27 bits and 28: one more digit of the sort, and no more than four."""
    import torch
    rng = np.random.default_rng(24)
    few = np.concatenate([rng.integers(0, vocab, size=12), [0, vocab - 1, vocab >> 1, (1 << 26) + 5, 5, vocab]])
    tokens = few[rng.integers(0, len(few), size=n)]
    grad = rng.integers(-8, 9, size=(n, 1)).astype(np.float64)      # (sums of few bits: exact)
    got = ap().april_embed_grad(place(grad, "f32"), index(tokens, 32), vocab)
    want = {int(t): grad[tokens == t, 0].sum() for t in few if t < vocab}
    for t, v in want.items():
        assert float(got[t, 0]) == v, t
    assert float(got.double().abs().sum()) == sum(abs(v) for v in want.values())


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_large_gradients_of_the_entropy_leave_masked_tokens_alone(t):
    """The gradient is linear in the entropy's own, and by a power of two to the bit: also where a logit is masked, at 2^60."""
    rng = np.random.default_rng(25)
    x = rng.standard_normal((9, 3001))
    x[:, 1::3] = -np.inf
    x[:, 2::7] = -3e38
    logits, tokens = place(x, t), index(np.zeros(9), 64)
    got = ap().april_logprobs(logits, tokens, entropy=True)
    one, large = (ap().april_logprobs_grad(logits, tokens, got, grad_entropy=f32(np.full(9, h))) for h in (1.0, 2.0 ** 60))
    assert np.array_equal(host(one) * 2.0 ** 60, host(large))
    assert (host(large)[x < -1e30] == 0).all() and (host(large) != 0).sum() > 9 * 1000


def test_a_written_out_is_known_to_autograd():
    """What is overwritten after autograd kept it makes the backward pass an error, not a wrong gradient."""
    import torch
    tokens, ids = index([1, 0, 2, -1], 64), index([[0], [1], [1], [0]], 32)
    rows = ap().april_expert_sort(ids, 2)
    table, x = f32(np.ones((5, 8))), f32(np.ones((4, 8)))
    logits = f32(np.ones((4, 8)))
    made = ap().april_logprobs(logits, tokens)
    for call in (lambda out: ap().april_embed(table, tokens, out=out), lambda out: ap().april_expert_gather(x, rows, out=out), lambda out: ap().april_expert_combine(x, rows, out=out),
                 lambda out: ap().april_embed_grad(x, tokens, 4, out=out), lambda out: ap().april_embed_grad(x, tokens, 4, out=out, accumulate=True),
                 lambda out: ap().april_logprobs_grad(logits, tokens, made, grad_logprob=f32(np.ones(4)), out=out)):
        kept = torch.zeros((4, 8), device="cuda")
        leaf = torch.ones((4, 8), device="cuda", requires_grad=True)
        y = (leaf * kept).sum()
        assert call(kept) is kept
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_logprobs_of_as_many_rows_as_31_bits_count():
    """One row of logits, repeated 2^31 - 1 times, nearly all padding: workgroups take a row every 2^20, and the last ones' next would be 2^31 and more."""
    import torch
    n = 2 ** 31 - 1
    rows = [0, 1, 2 ** 20, 2 ** 30 + 7, n - 2 ** 20 - 1, n - 2 ** 20, n - 1]
    x = np.array([[0.25, -1.5, 3.0]])
    tokens = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    tokens[rows] = torch.arange(len(rows), dtype=torch.int32, device="cuda") % 3
    got = ap().april_logprobs(f32(x).expand(n, 3), tokens)
    want = tr.logprobs(np.repeat(x, len(rows), 0), host(tokens[rows]))[0]
    near(host(got.logprob[rows]), want, U * (2 * np.log(3) + 3 + 48) + 4 * U * 5)
    assert int(torch.count_nonzero(got.logprob)) == len(rows)
    assert int(torch.count_nonzero(got.norm[:, 0])) == len(rows)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("parts", ["g", "gz", "h", "ghz"])
@pytest.mark.parametrize("temperature,size", [(1e-36, 1.0), (1e-30, 1e6), (1e-30, 1e12), (5e-39, 5.0)])
def test_gradients_at_small_temperatures(temperature, size, parts, t):
    """Gradients that are infinite over the temperature, or nearly: tokens of probability 0 (masked ones, and all but the largest here) have none, certain ones neither."""
    rng = np.random.default_rng(26)
    n, vocab = 24, 1003
    x = np.round(4 * rng.standard_normal((n, vocab)))
    x[:, 5::9] = -np.inf
    x[:, 700] = 50.0
    x[::3, 20] = 50.0                                        # two equal ones
    tokens = np.where(np.arange(n) % 2, 700, 3)
    tokens[4] = -1
    logits = place(x, t)
    got = ap().april_logprobs(logits, index(tokens, 64), temperature=temperature, entropy=True)
    temperature = float(np.float32(temperature))
    g, h, z = (np.float32(size * rng.choice([-1.0, 1.0, 0.5], size=n)) if c in parts else None for c in "ghz")
    grad = ap().april_logprobs_grad(logits, index(tokens, 64), got, grad_logprob=None if g is None else f32(g), grad_entropy=None if h is None else f32(h),
                                    grad_lse=None if z is None else f32(z), temperature=temperature)
    want, terms = tr.logprobs_grad(x, tokens, temperature, *(None if v is None else v.astype(np.float64) for v in (g, h, z)))
    # probabilities are 0, 1/2 and 1: what is left is a few products and differences, the log of 2, 1 / T, and bf16
    tol = 16 * U * terms + half(t) * np.abs(want)
    if h is not None and size / temperature > 1e37:          # (a difference of two equal numbers of that size: what rounding leaves of it may be infinite, too)
        pair = (np.arange(n) % 3 == 0)[:, None] & (x == 50.0)
        want, tol, grad = (np.where(pair, 0.0, v) for v in (want, tol, host(grad)))
        near(grad, want, tol, "gradient")
    else:
        near(host(grad), want, tol, "gradient")


def test_no_tangent_is_lost_in_a_backward_pass():
    """Forward mode over a recorded backward pass: refused where a tangent reaches it, right where none does."""
    import torch
    import torch.autograd.forward_ad as fw
    x, t, rows = f32(np.ones((4, 8))), index([1, 0, 2, -1], 64), ap().april_expert_sort(index([[0], [1], [1], [0]], 32), 2)
    w = f32(np.ones((4, 1)))
    for call in (lambda v: ap().april_logprobs(v, t).logprob, lambda v: ap().april_embed(v, t), lambda v: ap().april_expert_gather(v, rows), lambda v: ap().april_expert_combine(v, rows, w)):
        leaf = x.clone().requires_grad_()
        y = call(leaf)
        with fw.dual_level():
            dual = fw.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(Exception, match="has a tangent"):
                torch.autograd.grad((y * dual).sum(), leaf, retain_graph=True)
            (g,) = torch.autograd.grad(y.sum(), leaf)
            assert fw.unpack_dual(g).tangent is None and g.shape == x.shape


def test_saved_tensors_are_checked_again():
    """Hooks for saved tensors may give back others than were kept.  Those that serve are read as they are; other types, layouts, places or sizes are refused."""
    import torch
    rng = np.random.default_rng(27)
    n, d, e, k = 12, 16, 4, 2
    t, ids = index(rng.integers(0, d, size=n), 64), index(rng.integers(0, e, size=(n, k)), 32)
    rows, x, w = ap().april_expert_sort(ids, e, align=4), f32(rng.standard_normal((n, d))), f32(rng.random((n, k)))
    y, table, g = f32(rng.standard_normal((rows.source.shape[0], d))), f32(rng.standard_normal((d, 6))), f32(rng.standard_normal(n))

    def wide(v):
        """The same values in rows that lie apart (a matrix of floats; as they are, others)."""
        return torch.stack([v, v], 1).view(2 * v.shape[0], v.shape[1])[::2] if v.dim() == 2 and v.shape[1] == d else v

    def float16(v):
        return v.half() if v.is_floating_point() else v

    def turned(v):
        return v.t().contiguous().t() if v.dim() == 2 else v.repeat_interleave(2)[::2]

    def away(v):
        return v.cpu()

    def fewer(v):
        return v[:-1].contiguous()

    def counted(v):
        return v if v.is_floating_point() else v.short()

    def grads(leaves, call, hook):
        leaves = [v.clone().requires_grad_() for v in leaves]
        with torch.autograd.graph.saved_tensors_hooks(lambda v: v, hook):
            got = call(*leaves)
        return torch.autograd.grad(got, leaves, [(g if v.dim() == 1 else g[:, None]).expand(v.shape) if v.shape[0] == n else torch.ones_like(v) for v in got])

    def scored(v):
        got = ap().april_logprobs(v, t, entropy=True)
        return got.logprob, got.entropy
    for leaves, call, kinds in (((x,), scored, (float16, turned, away, fewer, counted)), ((table,), lambda v: (ap().april_embed(v, t),), (turned, away, fewer, counted)),
                                ((x,), lambda v: (ap().april_expert_gather(v, rows),), (turned, away, fewer, counted)),
                                ((y, w), lambda v, u: (ap().april_expert_combine(v, rows, u),), (float16, turned, away, fewer, counted))):
        for a, b in zip(grads(leaves, call, wide), grads(leaves, call, lambda v: v)):
            assert torch.equal(a, b)
        for hook in kinds:
            with pytest.raises(RuntimeError):                # (fewer rows of positions: torch refuses the gradient's shape, else the operator)
                grads(leaves, call, hook)


@pytest.mark.parametrize("weighted", [False, True])
def test_packed_rows_are_kept_for_the_weights_gradient_alone(weighted):
    """Without a gradient of the weights, what the experts made is not held until the backward pass and may be overwritten."""
    import torch
    rng = np.random.default_rng(28)
    n, k, e, d = 30, 2, 5, 24
    rows = ap().april_expert_sort(index(expert_ids(rng, n, k, e, True), 32), e, align=4)
    w = f32(rng.random((n, k))) if weighted else None
    base, g = f32(rng.standard_normal((rows.source.shape[0], d))).requires_grad_(), f32(rng.standard_normal((n, d)))
    kept = []
    packed = base * 2.0
    with torch.autograd.graph.saved_tensors_hooks(lambda v: kept.append(v.data_ptr()) or v, lambda v: v):
        out = ap().april_expert_combine(packed, rows, w)
    assert packed.data_ptr() not in kept
    with torch.no_grad():
        packed.fill_(float("nan"))
    (got,) = torch.autograd.grad(out, base, g)
    want, none = ap().april_expert_combine_grad(g, torch.zeros_like(base), rows, w, of_weights=False)
    assert none is None and torch.equal(got, want * 2.0)
    u = f32(rng.random((n, k))).requires_grad_()
    packed = base.detach() * 2.0
    out = ap().april_expert_combine(packed, rows, u)
    packed.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


STREAMED = [("bf16", 135000, 1000, 64, 0), ("bf16", 15001, 9001, 64, 20), ("bf16", 6800, 20000, 256, 0), ("bf16", 6803, 20001, 256, 40), ("bf16", 1950, 70000, 512, 9),
            ("f32", 75000, 900, 64, 0), ("f32", 13501, 5001, 64, 20), ("f32", 3400, 20000, 256, 5), ("f32", 1700, 40000, 512, 0), ("f32", 1701, 40001, 512, 30)]


@pytest.mark.parametrize("t,n,vocab,threads,top", STREAMED)
def test_logprobs_and_gradient_of_arrays_past_the_last_cache(t, n, vocab, threads, top):
    """Logits of more than 256 MB, whose accesses are streamed, in workgroups of 64, 256 and 512 threads: 48 rows against the plain form, the others copies of them, with the same bits at like
    addresses.

    A thread adds up V / threads exponentials one after another, and goes over to a new reference at most once for every 32 of them, two roundings each; 6 additions join a wavefront, threads / 64
    those."""
    import torch
    assert n * vocab * (2 if t == "f32" else 1) > 128 << 20
    rng = np.random.default_rng([n, vocab, top])
    few = place(hard_logits(rng, 48, vocab, t), t)
    tokens = rng.integers(0, vocab, size=48)
    tokens[[5, 30]] = -1, vocab
    of = rng.integers(0, 48, size=n)
    of[:48] = np.arange(48)
    at = torch.as_tensor(of).cuda()
    logits, idx = few[at], index(tokens[of], 64)
    got = ap().april_logprobs(logits, idx, entropy=True, lse=True, top=top)
    x = host(few)
    lp, ent, lse, best, ids = tr.logprobs(x, tokens, 1.0, top)
    chain = vocab / threads * (1 + 2 / 32) + 6 + threads / 64
    m = np.max(np.where(np.isfinite(x), x, -np.inf), axis=1, keepdims=True)
    with np.errstate(invalid="ignore", over="ignore"):
        dist = np.array([(m[r, 0] - x[r, k]) if 0 <= k < vocab else 0.0 for r, k in enumerate(tokens)])
        base = U * (2 * np.log(vocab) + chain + 48)
        near(host(got.logprob[:48]), lp, base + 4 * U * np.abs(dist), "logprob")
        near(host(got.entropy[:48]), ent, base * (2 + np.log(vocab)), "entropy")
        near(host(got.lse[:48]), lse, base + 4 * U * np.abs(lse), "lse")
        if top:
            assert np.array_equal(host(got.top_ids[:48]), ids)
            near(host(got.top_logprobs[:48]), best, base + 4 * U * np.abs(best), "top")
    first, per = {}, 8 if t == "bf16" else 4                 # (a row's sums go by its place to a 16-byte border)
    same = torch.as_tensor([first.setdefault((of[r], r * vocab % per), r) for r in range(n)]).cuda()
    alike = lambda v: torch.equal(v.nan_to_num(nan=123.0), v[same].nan_to_num(nan=123.0))  # noqa: E731
    assert all(alike(v) for v in got if v is not None)
    plain = ap().april_logprobs(logits, idx, top=top)        # (without the entropy's sum: the rest as with it)
    for a, b in zip(plain, got):
        assert a is None or torch.equal(a.nan_to_num(nan=123.0), b.nan_to_num(nan=123.0))
    g, h, z = (rng.standard_normal(48).astype(np.float32) for _ in range(3))
    finite = np.isfinite(x).any(axis=1) & ~np.isnan(x).any(axis=1) & ~(x == np.inf).any(axis=1)
    keep = finite | (tokens < 0)
    with np.errstate(invalid="ignore", over="ignore"):
        dist = np.minimum(np.abs(np.nan_to_num(m - x, nan=0.0, posinf=0.0, neginf=0.0)), 200.0)
    for with_entropy in (True, False):
        want, size = tr.logprobs_grad(x, tokens, 1.0, g.astype(np.float64), h.astype(np.float64) if with_entropy else None, z.astype(np.float64))
        grad = ap().april_logprobs_grad(logits, idx, got, grad_logprob=f32(g)[at], grad_entropy=f32(h)[at] if with_entropy else None, grad_lse=f32(z)[at])
        # each term: an exponential of that distance, the forward's log of the sum and entropy, a handful of products
        rel = U * (6 * dist + 4 * np.log(vocab) + chain + 64) * (3 if with_entropy else 1)
        tol = size * rel + half(t) * np.abs(want) + 1e-37 * (1 + np.nan_to_num(size)) + (2.0 ** -133 if t == "bf16" else 2.0 ** -149)
        near(host(grad[:48])[keep], want[keep], tol[keep], "gradient")
        assert alike(grad) and bool(grad[:48][torch.as_tensor(~keep).cuda()].isnan().all())
