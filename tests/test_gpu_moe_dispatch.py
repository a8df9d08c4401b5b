"""Prefill of routed experts in passes of more than 4096 assignments: the dispatch is april_expert_sort's then."""
import numpy as np
import pytest

import april_inputs as ai
from gpu_common import class_forced_tokens, have_gpu, make_engine, run_gpu
from test_gpu_moe import moe_parity

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not have_gpu():
        pytest.skip("no GPU")


@pytest.mark.parametrize("experts,top_k,prompts,length", [(32, 4, 60, 41), (256, 8, 30, 37), (96, 1, 70, 65)])
def test_prefill_against_the_oracle(experts, top_k, prompts, length):
    assert prompts * length * top_k > 4096
    shape = ai.ModelShape(1, 128, 4, 2, 32, 0, 512, n_experts=experts, experts_per_tok=top_k, d_expert_ffn=32)
    w = ai.Workload("moe_prefill", shape, prompts, length, prompts, prompts, 3, 1.0, 0.2, 2, 3, ai.SAMPLER_GREEDY, 0, 1, 29)
    moe_parity(w, 1, prompts, min_rows=prompts // 2)


def test_a_prompt_in_a_large_pass_has_the_bits_of_a_small_one():
    """200 rollouts of 5 prompts in one pass (16400 assignments), and 5 alone in one of 410, which one workgroup dispatches."""
    import paper_2509_18521_amd as ap
    shape = ai.ModelShape(2, 128, 4, 2, 32, 0, 512, n_experts=32, experts_per_tok=2, d_expert_ffn=64)
    rows = {}
    for n in (200, 5):
        w = ai.Workload("moe_pass", shape, 5, 41, n, n, 2, 1.0, 0.1, 2, 2, ai.SAMPLER_GREEDY, 0, 1, 31)
        reqs = ai.make_requests(w, n)
        tokens = class_forced_tokens(w, 5)
        ctx = make_engine(w, ai.make_weights(shape, w.seed), debug=True)
        try:
            for r in reqs:
                ap.april_debug_watch(ctx, r.request_id, 0, 2)
            run_gpu(ctx, reqs, n, n, 2, 1, forced={r.request_id: tokens[r.request_id % 5][:2] for r in reqs})
            rows[n] = {(r.request_id, i): ap.april_debug_logits(ctx, r.request_id, i, 512)[0] for r in reqs for i in range(2)}
        finally:
            ap.april_destroy(ctx)
    for (rid, i), row in rows[200].items():
        assert np.isfinite(row).all() and np.array_equal(row, rows[200][(rid % 5, i)]), (rid, i)
    for at, row in rows[5].items():
        assert np.max(np.abs(row - rows[200][at])) <= 2e-2 * max(1.0, np.max(np.abs(row))), at      # (other tiles of the projections)


@pytest.mark.parametrize("n", [6, 60])
@pytest.mark.parametrize("experts,top_k", [(32, 2), (96, 1), (256, 8)])
def test_a_prompt_of_nan_leaves_the_others_alone(experts, top_k, n):
    """A row of the embedding is NaN, as a policy that diverged may have it: its prompt's router rows have no largest expert.  Its logits are NaN; the other prompts' have the bits of a run
    without it, in passes that one workgroup dispatches and in sorted ones."""
    import paper_2509_18521_amd as ap
    shape = ai.ModelShape(2, 128, 4, 2, 32, 0, 512, n_experts=experts, experts_per_tok=top_k, d_expert_ffn=64)
    length = 4500 // (60 * top_k) + 20
    assert 6 * length * top_k <= 4096 < 60 * length * top_k
    w = ai.Workload("moe_nan", shape, n, length, n, n, 3, 1.0, 0.1, 3, 3, ai.SAMPLER_GREEDY, 0, 1, 37)
    weights, reqs, tokens = ai.make_weights(shape, w.seed), ai.make_requests(w, n), class_forced_tokens(w, n)
    lost, own = n // 2, 300                                  # the prompt, and the token that it alone has
    for r in reqs:
        r.tokens[r.tokens == own] = 7
    tokens[tokens == own] = 8
    reqs[lost].tokens[length // 3] = own
    rows = []
    for value in (None, np.nan):
        if value is not None:
            weights["tok_emb"] = weights["tok_emb"].copy()
            weights["tok_emb"][own] = value
        ctx = make_engine(w, weights, debug=True)
        try:
            for r in reqs:
                ap.april_debug_watch(ctx, r.request_id, 0, 3)
            run_gpu(ctx, reqs, n, n, 3, 1, forced={r.request_id: tokens[r.request_id] for r in reqs})
            rows.append({(r.request_id, i): ap.april_debug_logits(ctx, r.request_id, i, 512)[0] for r in reqs for i in range(3)})
        finally:
            ap.april_destroy(ctx)
    for (rid, i), row in rows[0].items():
        assert np.isfinite(row).all(), (rid, i)
        if rid == lost:
            assert np.isnan(rows[1][rid, i]).all(), i
        else:
            assert np.array_equal(row, rows[1][rid, i]), (rid, i)


def test_the_sort_and_the_one_workgroup_dispatch_give_the_same_bits():
    """The same prompts in a prefill of 4018 assignments, which one workgroup dispatches, and of 4100, which are sorted: experts' rows lie otherwise in their batches, nothing else differs."""
    import paper_2509_18521_amd as ap
    shape = ai.ModelShape(2, 128, 4, 2, 32, 0, 512, n_experts=32, experts_per_tok=2, d_expert_ffn=64)
    rows = []
    for n in (49, 50):
        w = ai.Workload("moe_border", shape, 50, 41, n, n, 2, 1.0, 0.1, 2, 2, ai.SAMPLER_GREEDY, 0, 1, 41)
        reqs = ai.make_requests(w, n)
        tokens = class_forced_tokens(w, 50)
        ctx = make_engine(w, ai.make_weights(shape, w.seed), debug=True, max_inflight=60)
        try:
            for r in reqs:
                ap.april_debug_watch(ctx, r.request_id, 0, 2)
            run_gpu(ctx, reqs, n, n, 2, 1, forced={r.request_id: tokens[r.request_id][:2] for r in reqs})
            rows.append({r.request_id: ap.april_debug_logits(ctx, r.request_id, 0, 512)[0] for r in reqs})
        finally:
            ap.april_destroy(ctx)
    assert len(rows[0]) == 49
    for rid, row in rows[0].items():
        assert np.isfinite(row).all() and np.array_equal(row, rows[1][rid]), rid
