"""Refusals of the scoring and training operators: found on the host, before anything is enqueued (no GPU needed)."""
import ctypes as C

import pytest

import paper_2509_18521_amd as ap

P, Q, R = 1 << 30, 1 << 32, 1 << 34             # addresses that are never read: every call here is refused first
NAN, INF = float("nan"), float("inf")

GOOD = dict(
    logprobs=dict(n_rows=3, vocab=100, dtype=1, index_bits=64, n_top=5, temperature=1.0, logits_row=100, logits=P, tokens=R, logprob=R, entropy=R, lse=R, norm=R, top_logprobs=R,
                  top_ids=R, workspace=R, workspace_bytes=1 << 40, stream=None),
    logprobs_grad=dict(n_rows=3, vocab=100, dtype=1, index_bits=64, temperature=1.0, reserved=0, logits_row=100, grad_row=100, logits=P, tokens=R, norm=R, entropy=R, grad_logprob=R,
                       grad_entropy=R, grad_lse=R, grad=Q, stream=None),
    embed=dict(n_rows=3, vocab=100, d=64, table_dtype=1, out_dtype=0, index_bits=32, scale=1.0, reserved=0, table_row=64, out_row=64, table=P, tokens=R, out=Q, stream=None),
    embed_grad=dict(n_rows=3, vocab=100, d=64, out_dtype=1, table_dtype=0, index_bits=32, scale=1.0, accumulate=0, out_row=64, table_row=64, grad_out=P, tokens=R, grad_table=Q,
                    workspace=R, workspace_bytes=1 << 40, stream=None),
    expert_sort=dict(n_rows=3, k=2, n_experts=4, align=1, n_packed=6, index_bits=32, ids=P, starts=P, source=P, position=P, workspace=R, workspace_bytes=1 << 40, stream=None),
    expert_gather=dict(n_rows=3, k=2, d=64, n_packed=6, dtype=1, reserved=0, x_row=64, packed_row=64, x=P, source=R, position=R, packed=Q, stream=None),
    expert_combine=dict(n_rows=3, k=2, d=64, n_packed=6, dtype=1, reserved=0, packed_row=64, out_row=64, packed=P, position=R, weights=R, out=Q, stream=None),
    expert_combine_grad=dict(n_rows=3, k=2, d=64, n_packed=6, dtype=1, reserved=0, out_row=64, packed_row=64, grad_packed_row=64, grad_out=P, packed=P, source=R, position=R, weights=R,
                             grad_packed=Q, grad_weights=R, stream=None),
)
BAD = dict(
    logprobs=[dict(n_rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dtype=2), dict(dtype=-1), dict(index_bits=16), dict(n_top=-1), dict(n_top=65), dict(n_top=101),
              dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-39), dict(temperature=3e38), dict(logits=None),
              dict(tokens=None), dict(top_ids=None), dict(top_logprobs=None), dict(logits=P + 1), dict(dtype=0, logits=P + 2), dict(tokens=R + 4), dict(norm=R + 4),
              dict(entropy=R + 2), dict(lse=R + 1), dict(logprob=R + 2), dict(top_ids=R + 2)],
    logprobs_grad=[dict(n_rows=-1), dict(vocab=0), dict(dtype=2), dict(index_bits=8), dict(reserved=1), dict(temperature=0.0), dict(temperature=NAN), dict(logits=None), dict(tokens=None),
                   dict(norm=None), dict(grad=None), dict(entropy=None), dict(grad=Q + 1), dict(logits=P + 1), dict(norm=R + 4), dict(grad_lse=R + 2), dict(grad_row=99),
                   dict(grad_row=-99), dict(grad_row=0), dict(grad=P + 2), dict(grad=P, grad_row=101), dict(grad=P + 2 * 199), dict(grad=P - 2 * 99),
                   dict(logits_row=200, grad_row=200, grad=P + 2 * 99), dict(logits_row=200, grad_row=200, grad=P + 2 * 101), dict(logits_row=0, grad=P)],
    embed=[dict(n_rows=-1), dict(vocab=0), dict(d=0), dict(d=(1 << 24) + 1), dict(table_dtype=2), dict(out_dtype=3), dict(index_bits=0), dict(scale=NAN), dict(scale=INF),
           dict(reserved=7), dict(table=None), dict(tokens=None), dict(out=None), dict(out=Q + 2), dict(table=P + 1), dict(tokens=R + 2), dict(out_row=63), dict(out_row=-1),
           dict(out=P + 4), dict(out=P + 64 * 2 * 99)],
    embed_grad=[dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(vocab=0), dict(d=0), dict(out_dtype=2), dict(table_dtype=2), dict(index_bits=1), dict(scale=INF),
                dict(accumulate=2), dict(grad_out=None), dict(tokens=None), dict(grad_table=None), dict(grad_table=Q + 2), dict(grad_out=P + 1), dict(table_row=63), dict(table_row=0),
                dict(grad_table=P + 64), dict(workspace=None), dict(workspace=R + 4), dict(workspace_bytes=100)],
    expert_sort=[dict(n_rows=-1), dict(k=0), dict(k=65), dict(n_rows=1 << 30, k=2, n_packed=2 ** 31 - 1), dict(n_experts=0), dict(n_experts=512), dict(align=0), dict(align=4097),
                 dict(n_packed=5), dict(align=4, n_packed=15), dict(n_packed=-1), dict(index_bits=31), dict(ids=None), dict(starts=None), dict(source=None), dict(position=None),
                 dict(ids=P + 2), dict(index_bits=64, ids=P + 4), dict(source=P + 1)],
    expert_gather=[dict(n_rows=-1), dict(k=0), dict(d=0), dict(n_packed=-1), dict(dtype=2), dict(reserved=1), dict(x=None), dict(source=None), dict(position=None), dict(packed=None),
                   dict(x=P + 1), dict(packed=Q + 1), dict(source=R + 2), dict(packed_row=63), dict(packed=P + 2)],
    expert_combine=[dict(n_rows=-1), dict(k=65), dict(d=0), dict(n_packed=-1), dict(dtype=9), dict(reserved=1), dict(packed=None), dict(position=None), dict(out=None), dict(packed=P + 1),
                    dict(out=Q + 1), dict(weights=R + 2), dict(out_row=1), dict(out=P + 128 * 5)],
    expert_combine_grad=[dict(n_rows=-1), dict(k=0), dict(d=1 << 25), dict(n_packed=-1), dict(dtype=2), dict(reserved=1), dict(grad_out=None), dict(packed=None), dict(source=None),
                         dict(position=None), dict(grad_out=P + 1), dict(grad_packed=Q + 1), dict(grad_weights=R + 2), dict(grad_packed_row=60), dict(grad_packed=P)],
)


def refused(name, **over):
    assert set(over) <= set(GOOD[name])
    args = getattr(ap, "april_%s_args" % name)(**{**GOOD[name], **over})
    lib = ap.load_library()
    assert getattr(lib, "april_" + name)(C.byref(args)) == ap.APRIL_EINVAL
    message = lib.april_last_error(None).decode()
    assert message.startswith("april_%s: " % name)
    return message


@pytest.mark.parametrize("name,over", [(n, o) for n, many in BAD.items() for o in many])
def test_refused(name, over):
    refused(name, **over)


@pytest.mark.parametrize("name", sorted(GOOD))
def test_null(name):
    lib = ap.load_library()
    assert getattr(lib, "april_" + name)(None) == ap.APRIL_EINVAL
    if hasattr(ap, "april_%s_args" % name) and "april_%s_workspace" % name in ap.EXPORTS:
        assert getattr(lib, "april_%s_workspace" % name)(None) == ap.APRIL_EINVAL


def test_workspace():
    lib = ap.load_library()
    for name in ("logprobs", "embed_grad", "expert_sort"):
        query = getattr(lib, "april_%s_workspace" % name)
        args = getattr(ap, "april_%s_args" % name)
        assert query(C.byref(args(**GOOD[name]))) >= 0
        assert query(C.byref(args(**{**GOOD[name], "n_rows": -1}))) == ap.APRIL_EINVAL
        assert query(C.byref(args(**{**GOOD[name], "n_rows": 0, **({"n_packed": 0} if name == "expert_sort" else {})}))) >= 0
        need = query(C.byref(args(**GOOD[name])))
        for over in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=R + 8)) if need else ():
            assert "workspace" in refused(name, **over)
    for name, sizes in (("embed_grad", dict(n_rows=1 << 30, d=1 << 24, vocab=1 << 30)), ("logprobs", dict(n_rows=2 ** 31 - 1, vocab=1 << 30, n_top=64)),
                        ("expert_sort", dict(n_rows=2 ** 31 - 5000, k=1, n_packed=2 ** 31 - 1))):
        args = getattr(ap, "april_%s_args" % name)(**{**GOOD[name], **sizes})
        assert getattr(lib, "april_%s_workspace" % name)(C.byref(args)) >= 0       # (counted in 64 bits)


def elements(p, n, row, length, size):
    return {p + (i * row + j) * size + b for i in range(n) for j in range(length) for b in range(size)}


def test_overlap_by_listing_bytes():
    """A gradient beside the logits in one wider array is taken, one that shares a byte with them is refused; where the strides differ, arrays whose
    addresses interleave are refused too."""
    refusals = 0
    for rows in (1, 2, 4):
        for row in (6, 7, 12, 13, 20):
            for grad_row in (6, 7, 12, 13, 20):
                for off in range(-60, 61, 3):
                    sizes = dict(n_rows=rows, vocab=6, dtype=1, logits=P, logits_row=row, grad=P + 2 * off, grad_row=grad_row)
                    a, b = elements(P, rows, row, 6, 2), elements(P + 2 * off, rows, grad_row, 6, 2)
                    same = off == 0 and (rows == 1 or row == grad_row)
                    if (a & b) and not same:
                        assert "overlaps" in refused("logprobs_grad", **sizes)
                        refusals += 1
    assert refusals > 200


def test_python_refusals():
    """What the binding finds itself, on tensors that are on no GPU or of the wrong kind."""
    import torch
    x, t = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int64)
    made = ap.Logprobs(None, None, None, None, None, torch.zeros((3, 2)))
    rows = ap.ExpertRows(torch.zeros(3, dtype=torch.int32), torch.zeros(6, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
    for call in (lambda: ap.april_logprobs(x, t), lambda: ap.april_logprobs(x[0], t), lambda: ap.april_logprobs_grad(x, t, made), lambda: ap.april_embed(x, t),
                 lambda: ap.april_embed_grad(x, t, 5), lambda: ap.april_expert_sort(t[:, None], 4), lambda: ap.april_expert_gather(x, rows),
                 lambda: ap.april_expert_combine(x, rows), lambda: ap.april_expert_combine_grad(x, x, rows)):
        with pytest.raises(ap.AprilError) as e:
            call()
        assert e.value.code == ap.APRIL_EINVAL
    y = x.clone().requires_grad_()
    for call in (lambda: ap.april_logprobs_grad(y, t, made), lambda: ap.april_embed_grad(y, t, 5), lambda: ap.april_embed(x, t, out=y), lambda: ap.april_embed(y, t, out=x),
                 lambda: ap.april_expert_gather(y, rows, out=x), lambda: ap.april_expert_combine(x, rows, out=y), lambda: ap.april_expert_combine_grad(x, y, rows)):
        with pytest.raises(ap.AprilError, match="requires a gradient"):
            call()


def test_forward_mode_derivatives_are_refused_and_not_silently_zero():
    """A dual tensor requires no gradient and has an address: its tangent would be lost."""
    import torch
    import torch.autograd.forward_ad as fw
    t, c = torch.zeros(3, dtype=torch.int64), torch.zeros((3, 8))
    made = ap.Logprobs(None, None, None, None, None, torch.zeros((3, 2)))
    rows = ap.ExpertRows(torch.zeros(3, dtype=torch.int32), torch.zeros(6, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
    bf16, pool = torch.bfloat16, torch.zeros((2, 2, 544), dtype=torch.uint8)
    q, table, lens = torch.zeros((3, 2, 32), dtype=bf16), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with fw.dual_level():
        x, w, d = (fw.make_dual(v, torch.ones_like(v)) for v in (c, torch.zeros((3, 2)), q))
        y = fw.make_dual(c.clone().requires_grad_(), torch.ones_like(c))
        g = fw.make_dual(torch.zeros(3), torch.ones(3))
        calls = [("logits", lambda: ap.april_logprobs(x, t)), ("logits", lambda: ap.april_logprobs(y, t)), ("table", lambda: ap.april_embed(x, t)), ("out", lambda: ap.april_embed(c, t, out=x)),
                 ("x", lambda: ap.april_expert_gather(x, rows)), ("out", lambda: ap.april_expert_gather(c, rows, out=x)), ("packed", lambda: ap.april_expert_combine(x, rows)),
                 ("weights", lambda: ap.april_expert_combine(c, rows, w)), ("out", lambda: ap.april_expert_combine(c, rows, out=x)),
                 ("logits", lambda: ap.april_logprobs_grad(x, t, made)), ("grad_logprob", lambda: ap.april_logprobs_grad(c, t, made, grad_logprob=g)),
                 ("grad_entropy", lambda: ap.april_logprobs_grad(c, t, made, grad_entropy=g)), ("grad_lse", lambda: ap.april_logprobs_grad(c, t, made, grad_lse=g)),
                 ("out", lambda: ap.april_logprobs_grad(c, t, made, out=x)), ("grad_out", lambda: ap.april_embed_grad(x, t, 5)), ("out", lambda: ap.april_embed_grad(c, t, 5, out=x)),
                 ("grad_out", lambda: ap.april_expert_combine_grad(x, c, rows)), ("packed", lambda: ap.april_expert_combine_grad(c, x, rows)),
                 ("weights", lambda: ap.april_expert_combine_grad(c, c, rows, w)),
                 ("q", lambda: ap.april_cache_attention(d, pool, table, lens, 60)), ("out", lambda: ap.april_cache_attention(q, pool, table, lens, 60, out=d)),
                 ("lse", lambda: ap.april_cache_attention(q, pool, table, lens, 60, lse=w)), ("k", lambda: ap.april_cache_append(pool, d, q, t)),
                 ("v", lambda: ap.april_cache_append(pool, q, d, t)), ("k_values", lambda: ap.april_cache_append(pool, q, q, t, k_values=d)),
                 ("v_values", lambda: ap.april_cache_append(pool, q, q, t, v_values=d))]
        for name, call in calls:
            for on in (torch.enable_grad, torch.no_grad):
                with on(), pytest.raises(ap.AprilError, match="^april error -1: %s has a tangent" % name):
                    call()
        with pytest.raises(ap.AprilError, match="not on a GPU"):        # a tensor without one goes on
            ap.april_logprobs(c, t)
        with pytest.raises(ap.AprilError, match="not on a GPU"):
            ap.april_logprobs(fw.unpack_dual(x).primal, t)


def test_tensors_of_other_dimensions_are_refused():
    import torch
    t, made = torch.zeros(3, dtype=torch.int64), ap.Logprobs(None, None, None, None, None, torch.zeros((3, 2)))
    rows = ap.ExpertRows(torch.zeros(3, dtype=torch.int32), torch.zeros(6, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32))
    for x in (torch.zeros(()), torch.zeros(3), torch.zeros((2, 3, 8))):
        for call in (lambda: ap.april_logprobs(x, t), lambda: ap.april_logprobs_grad(x, t, made), lambda: ap.april_embed(x, t), lambda: ap.april_embed_grad(x, t, 5),
                     lambda: ap.april_expert_sort(x, 4), lambda: ap.april_expert_gather(x, rows), lambda: ap.april_expert_combine(x, rows), lambda: ap.april_expert_combine_grad(x, x, rows)):
            with pytest.raises(ap.AprilError, match="two dimensions wanted"):
                call()
