"""Rollouts over the 4-bit KV cache (APRIL_DTYPE_BF16_KV4) against the oracle with the same rounding of keys and values."""
from dataclasses import replace

import numpy as np
import pytest

import april_inputs as ai
from gpu_common import assert_schedule_equal, have_gpu, make_engine, req_dicts, run_gpu, run_oracle
from oracle.model import Decoder

pytestmark = pytest.mark.gpu

# Keys and values of the two sides differ before rounding by the bf16 path's relative error d (at most 2^-8 of an operand, about 4e-3
# of a product); a code whose value lies within that of a rounding border flips, by a step s of about 0.3 of the block's deviation: the chance is
# d / s, the square of the error d s, so sqrt(4e-3 * 0.3) = 3.5 % of a deviation, at random.  That share of the attention's output
# passes to the residual stream, all of it at most (a context of one token: nothing is averaged): d = 3.5 % for the second layer's keys and
# values, whose codes then differ by sqrt(0.035 * 0.3) = 10 %, together sqrt(0.035^2 + 0.10^2) = 11 %.  The largest error of a vocabulary is as many
# deviations as its largest logit.  One layer: 3.5 %, and half again for the worst of some dozens of rows.
TOL = {1: 5e-2, 2: 0.11}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not have_gpu():
        pytest.skip("no GPU")


def ap():
    import paper_2509_18521_amd
    return paper_2509_18521_amd


def kv4(shape):
    return replace(shape, dtype=ai.DTYPE_BF16_KV4)


def parity(w, steps, n_requests, min_rows, **kw):
    """Schedule and tokens equal, logits of every forced token within TOL of the oracle's; and nearer to them than to those of an
    oracle without the rounding, which shows that the rounding is the stated one."""
    weights = ai.make_weights(w.shape, w.seed)
    reqs = ai.make_requests(w, n_requests)
    want, eng = run_oracle(w, weights, reqs, w.n_target, w.n_overprovision, w.max_new, steps, keep_logits=True)
    tokens = {}
    for o in want:
        tokens.update(dict(zip(o["ids"], o["tokens"])))
    tokens.update(want[-1]["buffer_tokens"])
    ctx = make_engine(w, weights, debug=True, **kw)
    try:
        for rid in tokens:
            ap().april_debug_watch(ctx, rid, 0, w.max_new)
        got = run_gpu(ctx, reqs, w.n_target, w.n_overprovision, w.max_new, steps, forced=tokens)
        assert_schedule_equal(got, want)
        plain = Decoder(w.shape, weights)
        plain.kv_round = None
        near, far, worst, rows = 0.0, 0.0, 0.0, 0
        for rid, toks in tokens.items():
            prompt = next(r.tokens for r in reqs if r.request_id == rid)
            whole = plain.forward_block(np.concatenate([prompt, toks[:-1]]).astype(np.int64), plain.new_cache())[len(prompt) - 1:] if rows < 40 else None
            for i in range(len(toks)):
                lg = ap().april_debug_logits(ctx, rid, i, w.shape.vocab)[0]
                ref = eng.logits[(rid, i)]
                worst = max(worst, float(np.max(np.abs(lg - ref))) / max(1.0, float(np.max(np.abs(ref)))))
                if whole is not None:
                    near += float(np.sum((lg - ref) ** 2))
                    far += float(np.sum((lg - whole[i]) ** 2))
                rows += 1
        assert rows >= min_rows
        assert worst <= TOL[w.shape.n_layers], worst
        assert near < 0.25 * far, (near, far)
    finally:
        ap().april_destroy(ctx)


@pytest.mark.parametrize("n_q,n_kv,dh,d_model", [(14, 2, 64, 896), (8, 2, 128, 256), (4, 4, 32, 128), (16, 1, 64, 192), (5, 1, 128, 160)])
def test_logits_of_forced_tokens(n_q, n_kv, dh, d_model):
    shape = kv4(ai.ModelShape(2, d_model, n_q, n_kv, dh, 256, 512))
    parity(ai.Workload("kv4", shape, 6, 70, 3, 5, 16, 2.2, 0.5, 4, 16, ai.SAMPLER_GREEDY, 0, 2, 5), 2, 9, 40)


def test_routed_experts():
    shape = kv4(ai.ModelShape(1, 128, 4, 2, 64, 0, 512, n_experts=32, experts_per_tok=8, d_expert_ffn=32))
    w = ai.Workload("kv4_moe", shape, 4, 20, 2, 3, 8, 1.6, 0.4, 3, 8, ai.SAMPLER_GREEDY, 0, 1, 9)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, 5)
    ctx = make_engine(w, weights)
    try:
        got = run_gpu(ctx, reqs, 2, 3, 8, 1)
        assert len(got[0]["ids"]) == 2 and all(len(t) > 0 for t in got[0]["tokens"])
        assert ap().april_get_info(ctx)["kv_bytes_per_token"] == 1 * 2 * 17 * 64 // 16
    finally:
        ap().april_destroy(ctx)


# A routing decision hangs on router probabilities, whose logits differ by the same share of a deviation as the normed residual stream: of the attention's
# output 3.5 % at most (above), times its own size beside the embedding's 1, the root of the weights' squares, about 0.3 over 20 tokens: 1 %.  Two of them,
# and the largest of some hundred decisions, three deviations: 4.2 %; and the bf16 path's 3 %.  Nearer decisions are not compared.
ROUTE_MARGIN = 7.5e-2


@pytest.mark.parametrize("n_q,n_kv,dh,experts,top_k,ffn", [(4, 2, 64, 32, 8, 32), (8, 2, 128, 64, 4, 64), (6, 3, 32, 32, 1, 96)])
def test_logits_of_routed_experts(n_q, n_kv, dh, experts, top_k, ffn):
    """One layer, whose keys and values no routing decision has touched: the logits of forced tokens, where the oracle's own decision is no near-tie."""
    shape = kv4(ai.ModelShape(1, 128, n_q, n_kv, dh, 0, 512, n_experts=experts, experts_per_tok=top_k, d_expert_ffn=ffn))
    w = ai.Workload("kv4_routed", shape, 6, 24, 3, 5, 14, 2.0, 0.5, 3, 14, ai.SAMPLER_GREEDY, 0, 2, 29)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, 10)
    want, eng = run_oracle(w, weights, reqs, w.n_target, w.n_overprovision, w.max_new, 2, keep_logits=True)
    tokens = {}
    for o in want:
        tokens.update(dict(zip(o["ids"], o["tokens"])))
    tokens.update(want[-1]["buffer_tokens"])
    dec = Decoder(shape, weights)
    prompt = {r.request_id: list(r.tokens) for r in reqs}
    ctx = make_engine(w, weights, debug=True)
    try:
        for rid in tokens:
            ap().april_debug_watch(ctx, rid, 0, w.max_new)
        assert_schedule_equal(run_gpu(ctx, reqs, w.n_target, w.n_overprovision, w.max_new, 2, forced=tokens), want)
        worst, rows, near_ties = 0.0, 0, 0
        for rid, toks in tokens.items():
            dec.route_margins = []
            dec.forward_block(prompt[rid] + list(toks[:-1]), dec.new_cache())
            tied = {p - (len(prompt[rid]) - 1) for p, _, m in dec.route_margins if m < ROUTE_MARGIN}
            for i in range(len(toks)):
                if i in tied:
                    near_ties += 1
                    continue
                ref = eng.logits[(rid, i)]
                worst = max(worst, float(np.max(np.abs(ap().april_debug_logits(ctx, rid, i, shape.vocab)[0] - ref))) / max(1.0, float(np.max(np.abs(ref)))))
                rows += 1
        print(f"routed experts over the 4-bit cache: rows {rows}, near-ties {near_ties}, worst {worst:.3g}")
        assert rows >= 15 and worst <= TOL[1], (rows, near_ties, worst)
    finally:
        ap().april_destroy(ctx)


@pytest.mark.parametrize("head_dim,prompt_len", [(64, 2100), (128, 4150)])
def test_contexts_of_several_splits(head_dim, prompt_len):
    shape = kv4(ai.ModelShape(1, 256, 256 // head_dim, 2, head_dim, 256, 512))
    parity(ai.Workload("kv4_long", shape, 3, prompt_len, 2, 3, 8, 1.6, 0.4, 3, 8, ai.SAMPLER_GREEDY, 0, 2, 77), 2, 5, 12)


@pytest.mark.parametrize("n_q,n_kv,dh,d_model,prompt_len", [(14, 2, 64, 896, 70), (8, 2, 128, 256, 1100), (16, 1, 128, 192, 31), (3, 3, 32, 160, 16)])
def test_rotary_inside_the_attention_or_before_it(n_q, n_kv, dh, d_model, prompt_len, monkeypatch):
    """Both sum the projection's partials in one order and round alike, so every logit is the same to the bit."""
    shape = kv4(ai.ModelShape(2, d_model, n_q, n_kv, dh, 256, 512))
    w = ai.Workload("kv4_rope", shape, 5, prompt_len, 5, 5, 24, 2.0, 0.5, 4, 24, ai.SAMPLER_GREEDY, 0, 1, 15)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, 5)
    logits = []
    for fused in ("1", "0"):
        monkeypatch.setenv("APRIL_FUSE_ROPE", fused)
        ctx = make_engine(w, weights, debug=True)
        try:
            for r in reqs:
                ap().april_debug_watch(ctx, r.request_id, 0, w.max_new)
            got = run_gpu(ctx, reqs, 5, 5, w.max_new, 1)[0]
            logits.append({(rid, i): ap().april_debug_logits(ctx, rid, i, shape.vocab)[0]
                           for rid, t in zip(got["ids"], got["tokens"]) for i in range(len(t))})
        finally:
            ap().april_destroy(ctx)
    assert len(logits[0]) >= 20 and logits[0].keys() == logits[1].keys()
    for at in logits[0]:
        np.testing.assert_array_equal(logits[0][at], logits[1][at])


def test_many_rows_in_flight():
    shape = kv4(ai.ModelShape(2, 128, 4, 2, 32, 256, 512))
    parity(ai.Workload("kv4_rows", shape, 40, 6, 100, 160, 5, 1.2, 0.4, 2, 5, ai.SAMPLER_GREEDY, 0, 1, 5), 1, 160, 300)


def test_tokens_do_not_depend_on_the_schedule():
    """Carried over with resident KV or run with N' = N, token for token; with the KV dropped the schedule stays, and what was
    generated before a rollout was first parked."""
    shape = kv4(ai.ModelShape(3, 128, 4, 2, 64, 256, 1024))
    w = ai.Workload("kv4_small", shape, 8, 37, 5, 9, 60, 3.0, 0.6, 3, 60, ai.SAMPLER_GREEDY, 0, 4, 31)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, ai.requests_needed(w))
    ctxs = [make_engine(w, weights) for _ in range(3)]

    def drop(ctx, buf):
        ap().april_buffer_drop_kv(ctx, buf)
        return buf
    try:
        a = run_gpu(ctxs[0], reqs, w.n_target, w.n_overprovision, w.max_new, w.steps)
        b = run_gpu(ctxs[1], reqs, w.n_target, w.n_overprovision, w.max_new, w.steps, between=drop)
        c = run_gpu(ctxs[2], reqs, w.n_target, w.n_target, w.max_new, w.steps)
    finally:
        for x in ctxs:
            ap().april_destroy(x)
    assert sum(g["res"].reprefill_tokens for g in b) > 0
    assert_schedule_equal(b, a)
    parked, ta, tb = {}, {}, {}
    for x, y in zip(a, b):
        for rid, toks in x["buffer_tokens"].items():
            parked.setdefault(rid, len(toks))
        ta.update(zip(x["ids"], x["tokens"]))
        tb.update(zip(y["ids"], y["tokens"]))
    assert ta.keys() == tb.keys() and parked
    for rid, toks in ta.items():
        keep = parked.get(rid, len(toks))
        assert tb[rid][:keep] == toks[:keep], rid
    tc = {rid: t for g in c for rid, t in zip(g["ids"], g["tokens"])}
    assert set(ta) & set(tc)
    for rid in set(ta) & set(tc):
        assert ta[rid] == tc[rid], rid


def test_a_small_pool_preempts_as_the_oracle_does():
    """Pages run out: the youngest rollouts are preempted and prefilled again, the schedule is the oracle's."""
    from oracle.scheduler import PagePool
    shape = kv4(ai.ModelShape(1, 64, 2, 1, 32, 64, 128))
    w = ai.Workload("kv4_pool", shape, 8, 20, 4, 8, 60, 3.2, 0.6, 8, 60, ai.SAMPLER_GREEDY, 0, 3, 3)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, ai.requests_needed(w))
    n_pages, page = 22, 16 * 1 * 17 * 32 // 16
    want, _ = run_oracle(w, weights, reqs, w.n_target, w.n_overprovision, w.max_new, w.steps, pool=PagePool(total=n_pages, page_tokens=16))
    ctx = make_engine(w, weights, kv_pool_bytes=n_pages * page)
    try:
        info = ap().april_get_info(ctx)
        assert info["kv_blocks_total"] == n_pages and info["kv_bytes_per_token"] == 34
        got = run_gpu(ctx, reqs, w.n_target, w.n_overprovision, w.max_new, w.steps)
    finally:
        ap().april_destroy(ctx)
    assert_schedule_equal(got, want)
    assert sum(g["n_preempted"] for g in got) == sum(o["n_preempted"] for o in want) > 0


@pytest.mark.parametrize("d_model,n_q,n_kv,head_dim", [(160, 5, 1, 32), (192, 6, 2, 64), (2048, 4, 2, 128)])
def test_sampling_rows_alone_behind_the_last_keys(d_model, n_q, n_kv, head_dim):
    """Prompts together in a pass whose last layer takes the sampling rows only, and each alone in one that takes all: the same bits."""
    shape = kv4(ai.ModelShape(2, d_model, n_q, n_kv, head_dim, 224, 512))
    weights = ai.make_weights(shape, 11)
    rng = np.random.default_rng(d_model)
    lengths = [1, 2, 31, 77]
    prompts = [rng.integers(0, shape.vocab, t, dtype=np.int32) for t in lengths + [5000]]
    w = ai.Workload("last", shape, 1, 5010, 8, 8, 3, 0.0, 0.1, 3, 1, ai.SAMPLER_GREEDY, 0, 1, 11)
    ctx = make_engine(w, weights, debug=True, max_inflight=8)

    def logits(ids, which):
        for i in ids:
            ap().april_debug_watch(ctx, i, 0, 3)
        reqs = [ai.Request(i, prompts[p], 3) for i, p in zip(ids, which)]
        ap().april_buffer_free(ctx, ap().april_rollout_step(ctx, req_dicts(reqs), len(ids), len(ids), 3).buffer)
        return [[ap().april_debug_logits(ctx, i, g, shape.vocab)[0] for g in range(3)] for i in ids]

    try:
        together = logits(range(len(prompts)), range(len(prompts)))
        for p in range(len(lengths)):
            alone = logits([100 + p], [p])[0]
            assert np.isfinite(alone[0]).all() and all(np.array_equal(x, y) for x, y in zip(alone, together[p])), lengths[p]
    finally:
        ap().april_destroy(ctx)


def test_paused_and_updated():
    """The cache's memory released and mapped again, the weights replaced: the rollouts go on, token for token as without it."""
    shape = kv4(ai.ModelShape(1, 128, 4, 2, 64, 128, 256))
    w = ai.Workload("kv4_pause", shape, 6, 20, 3, 5, 20, 2.4, 0.4, 6, 20, ai.SAMPLER_GREEDY, 0, 2, 3)
    weights = ai.make_weights(shape, w.seed)
    reqs = ai.make_requests(w, ai.requests_needed(w))
    outs = []
    for pause in (False, True):
        ctx = make_engine(w, weights, pausable=True)

        def between(c, buf):
            ap().april_buffer_drop_kv(c, buf)
            if pause:
                ap().april_memory_pause(c, ap().APRIL_MEM_KV)
                ap().april_memory_resume(c, ap().APRIL_MEM_KV)
                ap().april_update_weights(c, ap().pack_weights(shape, weights))
            return buf
        try:
            outs.append(run_gpu(ctx, reqs, w.n_target, w.n_overprovision, w.max_new, w.steps, between=between))
        finally:
            ap().april_destroy(ctx)
    assert [g["tokens"] for g in outs[0]] == [g["tokens"] for g in outs[1]]


@pytest.mark.parametrize("env", ["APRIL_GEMM", "APRIL_ATTN"])
def test_the_reference_kernels_do_not_take_it(env, monkeypatch):
    shape = kv4(ai.ModelShape(1, 64, 2, 1, 32, 64, 128))
    w = ai.Workload("kv4_ref", shape, 1, 4, 1, 1, 4, 1.0, 0.1, 1, 4, ai.SAMPLER_GREEDY, 0, 1, 3)
    monkeypatch.setenv(env, "ref")
    with pytest.raises(ap().AprilError) as e:
        make_engine(w, ai.make_weights(shape, 3))
    assert e.value.code == ap().APRIL_EINVAL
