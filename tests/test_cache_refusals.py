"""Refusals of the 4-bit cache's operators: found on the host, before anything is enqueued (no GPU needed)."""
import ctypes as C

import pytest

import paper_2509_18521_amd as ap
from paper_2509_18521_amd import binding

P = 1 << 20                                     # an address that is never read: every call here is refused first


def attention_args(**over):
    a = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, n_pages=9, n_seqs=3, max_pages=4, n_rows=3, max_q=1, max_len=60, scale=0.0, table_stride=4,
             q_row=512, q_head=64, out_row=512, out_head=64, q=P, pool=P, block_table=P, lens=P, q_start=None, out=P, lse=None, workspace=P,
             workspace_bytes=1 << 40, stream=None)
    assert set(over) <= set(a)
    return ap.april_cache_attention_args(**{**a, **over})


def append_args(**over):
    a = dict(n_pages=9, n_kv_heads=2, head_dim=64, n_rows=3, dtype=1, reserved=0, k_row=128, k_head=64, v_row=128, v_head=64, k=P, v=P, k_values=None,
             v_values=None, slot_map=P, pool=P, stream=None)
    assert set(over) <= set(a)
    return ap.april_cache_append_args(**{**a, **over})


def extend_args(**over):
    a = dict(n_seqs=3, max_pages=4, n_pages=9, n_rows=5, table_stride=4, lens=P, new_lens=P, free_top=P, block_table=P, free_pages=P, lens_out=P,
             free_top_out=P, q_start=P, slot_map=P, positions=P, status=P, stream=None)
    assert set(over) <= set(a)
    return ap.april_cache_extend_args(**{**a, **over})


def refused(call, args):
    rc = call(None if args is None else C.byref(args))
    assert rc == ap.APRIL_EINVAL
    return ap.load_library().april_last_error(None).decode()


@pytest.mark.parametrize("over", [
    dict(head_dim=80), dict(head_dim=0), dict(n_q_heads=7), dict(n_q_heads=34), dict(n_kv_heads=0), dict(n_q_heads=-8), dict(n_pages=0), dict(n_seqs=-1),
    dict(n_rows=-1), dict(max_pages=0), dict(max_q=0), dict(max_len=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(q=None), dict(pool=None), dict(block_table=None), dict(lens=None), dict(out=None), dict(n_rows=2), dict(q=P + 8), dict(q_row=513),
    dict(q_head=68), dict(pool=P + 8), dict(out=P + 4), dict(out_row=514), dict(table_stride=3)])
def test_attention(over):
    assert "april_cache_attention" in refused(ap.load_library().april_cache_attention, attention_args(**over))


def overlap(n, row, m, head, length):
    """By listing the elements."""
    seen = [i * row + j * head + d for i in range(n) for j in range(m) for d in range(length)]
    return len(set(seen)) < len(seen)


def test_attention_refuses_results_that_overlap():
    """Rows and heads in either order, interleaved, backwards, and alone (a stride is then not used), for all strides about a head's length."""
    call = ap.load_library().april_cache_attention
    refusals = 0
    for rows, heads in ((3, 2), (2, 4), (5, 3), (1, 4), (4, 1), (1, 1)):
        for row in (0, 28, 32, 36, 40, 64, 72, 96, 100, 128, 160, 1000, -32, -96, -28):
            for head in (0, 28, 32, 36, 48, 64, 68, 96, 128, 160, 192, 1000, -64, -20):
                # (another refusal comes behind this one: nothing is launched)
                args = attention_args(head_dim=32, n_q_heads=heads, n_kv_heads=1, n_rows=rows, n_seqs=2, q_start=P, out_row=row, out_head=head, table_stride=3)
                message = refused(call, args)
                assert ("heads of out overlap" in message) == overlap(rows, row, heads, head, 32), (rows, heads, row, head, message)
                refusals += "heads of out overlap" in message
    assert refusals > 200


@pytest.mark.parametrize("row,head,bad", [(1 << 62, 64, False), (-(1 << 62), 1 << 61, True), (-(1 << 63), -(1 << 63), True), (1 << 40, 1 << 40, True), (1 << 40, (1 << 40) + 32, True),
                                          (1 << 40, (1 << 40) + 64, False)])
def test_attention_of_large_strides(row, head, bad):
    assert ("heads of out overlap" in refused(ap.load_library().april_cache_attention, attention_args(out_row=row, out_head=head, table_stride=3))) == bad


def test_attention_needs_its_workspace():
    lib = ap.load_library()
    a = attention_args(max_pages=4096, table_stride=4096, max_len=60000)
    need = lib.april_cache_attention_workspace(C.byref(a))
    assert need >= 0
    if need:
        for over in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 4)):
            assert "workspace" in refused(lib.april_cache_attention, attention_args(max_pages=4096, table_stride=4096, max_len=60000, **over))
    assert "head_dim" in refused(lib.april_cache_attention_workspace, attention_args(head_dim=96))


# A launch has fewer than 2^32 threads in a dimension.  The largest that fits, the first that does not, and which of them it is:
# tiles of 256 columns, workgroups of 256 threads; sequences alone; their splits (two for 5000 tokens, 8 for 32768); the join's workgroup a row.
LAUNCHES = [(dict(n_q_heads=32, n_kv_heads=8, n_seqs=4096, max_len=2048, n_rows=1 << 20), "max_q", 511 * 64, 511 * 64 + 1),
            (dict(n_q_heads=32, n_kv_heads=8, n_seqs=2048, max_len=2048, n_rows=1 << 20), "max_q", 1023 * 64, 1023 * 64 + 1),
            (dict(n_q_heads=1, n_kv_heads=1, n_rows=1 << 25, max_len=60), "n_seqs", (1 << 24) - 1, 1 << 24),
            (dict(n_q_heads=4, n_kv_heads=4, n_rows=1 << 25, max_len=5000), "n_seqs", (1 << 21) - 1, 1 << 21),
            (dict(n_q_heads=4, n_kv_heads=4, n_rows=1 << 25, max_len=32768), "n_seqs", (1 << 19) - 1, 1 << 19),
            (dict(n_q_heads=1, n_kv_heads=1, n_rows=1 << 25, max_len=5000, max_q=64), "n_seqs", (1 << 18) - 1, 1 << 18),
            (dict(n_q_heads=65536, n_kv_heads=65536, n_rows=1 << 30, max_q=1 << 30, n_seqs=1 << 30), "max_len", None, 0)]


@pytest.mark.parametrize("sizes,name,fits,first", LAUNCHES)
def test_attention_larger_than_a_launch(sizes, name, fits, first):
    lib = ap.load_library()
    sizes = dict(dict(max_pages=4096, table_stride=4096), **sizes)
    if fits is not None:
        assert lib.april_cache_attention_workspace(C.byref(attention_args(**sizes, **{name: fits}))) >= 0
    args = attention_args(**sizes, **{name: first})
    for call in (lib.april_cache_attention_workspace, lib.april_cache_attention):
        assert "more work than one call takes" in refused(call, args)


@pytest.mark.parametrize("heads", [2, 8, 16])
def test_attention_columns_are_counted_in_31_bits(heads):
    """Rows times query heads of a KV head, up to whole tiles of 256; fewer workgroups than a launch takes."""
    lib = ap.load_library()
    most = ((1 << 31) - 256) // heads
    sizes = dict(n_q_heads=heads, n_kv_heads=1, head_dim=32, n_seqs=1, n_rows=(1 << 31) - 1, max_len=60, q_start=P)
    assert lib.april_cache_attention_workspace(C.byref(attention_args(max_q=most, **sizes))) == 0
    for rows in (most + 1, (1 << 31) - 1):
        for call in (lib.april_cache_attention_workspace, lib.april_cache_attention):
            assert "more work than one call takes" in refused(call, attention_args(max_q=rows, **sizes))


def test_long_contexts_of_many_rows_that_fit_a_launch():
    """2064384 workgroups: far below the limit, whatever the bounds on rows and length would allow together."""
    a = attention_args(n_q_heads=32, n_kv_heads=8, n_seqs=4096, max_q=4000, n_rows=1 << 20, max_len=32768, max_pages=4096, table_stride=4096)
    assert ap.load_library().april_cache_attention_workspace(C.byref(a)) == 0


@pytest.mark.parametrize("over", [
    dict(head_dim=48), dict(n_pages=0), dict(n_kv_heads=0), dict(n_rows=-1), dict(dtype=2), dict(reserved=1), dict(k=None), dict(v=None), dict(slot_map=None),
    dict(pool=None), dict(pool=P + 4), dict(slot_map=P + 4), dict(k=P + 1), dict(v=P + 1), dict(dtype=0, k=P + 2), dict(k_values=P + 8), dict(v_values=P + 8)])
def test_append(over):
    assert "april_cache_append" in refused(ap.load_library().april_cache_append, append_args(**over))


@pytest.mark.parametrize("rows", [(1 << 28) - 15, 1 << 30, (1 << 31) - 1])
def test_append_larger_than_a_launch(rows):
    assert "n_rows" in refused(ap.load_library().april_cache_append, append_args(n_rows=rows))


@pytest.mark.parametrize("over", [
    dict(n_seqs=0), dict(n_seqs=65537), dict(max_pages=0), dict(max_pages=(1 << 27) + 1), dict(n_pages=0), dict(n_rows=-1), dict(table_stride=3), dict(slot_map=P + 4)] +
    [{n: None} for n in ("lens", "new_lens", "free_top", "block_table", "free_pages", "lens_out", "free_top_out", "q_start", "slot_map", "positions", "status")])
def test_extend(over):
    assert "april_cache_extend" in refused(ap.load_library().april_cache_extend, extend_args(**over))


def test_null_arguments():
    lib = ap.load_library()
    for name in ("april_cache_extend", "april_cache_append", "april_cache_attention", "april_cache_attention_workspace"):
        assert "null argument" in refused(getattr(lib, name), None)


def test_nothing_to_do_is_no_error():
    lib = ap.load_library()
    assert lib.april_cache_append(C.byref(append_args(n_rows=0, k=None, v=None, slot_map=None))) == 0
    assert lib.april_cache_attention(C.byref(attention_args(n_rows=0, n_seqs=0, q=None, out=None))) == 0


def test_block_bytes():
    assert [ap.april_cache_block_bytes(d) for d in (32, 64, 128)] == [544, 1088, 2176]
    with pytest.raises(ap.AprilError) as e:
        ap.april_cache_block_bytes(256)
    assert e.value.code == ap.APRIL_EINVAL


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu_or_of_another_kind():
    import torch
    t = lambda *s, d=torch.int32: torch.zeros(s, dtype=d)  # noqa: E731
    with pytest.raises(ap.AprilError, match="not on a GPU"):
        ap.april_cache_extend(t(3), t(3), t(3, 4), t(9), t(1), 5)
    with pytest.raises(ap.AprilError, match="not on a GPU"):
        ap.april_cache_append(t(2, 2, 544, d=torch.uint8), t(3, 2, 32, d=torch.float32), t(3, 2, 32, d=torch.float32), t(3, d=torch.int64))
    with pytest.raises(ap.AprilError, match="not on a GPU"):
        ap.april_cache_attention(t(3, 2, 32, d=torch.bfloat16), t(2, 2, 544, d=torch.uint8), t(3, 4), t(3), 60)
    binding._need_torch()
    i32 = torch.int32
    for bad, match in ((t(3, d=torch.int64), "torch.int32 wanted"), (t(4), "shape"), (t(6)[::2], "contiguous")):
        with pytest.raises(ap.AprilError, match=match):
            binding._ptr("x", bad, i32, (3,), -1)               # (-1: what a tensor on the CPU calls its GPU)
    assert binding._ptr("x", t(3), i32, (3,), -1)
    with pytest.raises(ap.AprilError, match="on GPU 0"):
        binding._ptr("x", t(3), i32, (3,), 0)
    with pytest.raises(ap.AprilError, match="adjacent"):
        binding._table(t(4, 3).t(), 3, -1)
    with pytest.raises(ap.AprilError, match="rows"):
        binding._table(t(4, 3), 3, -1)
    with pytest.raises(ap.AprilError, match="adjacent"):
        binding._rows("x", t(3, 32, 2).transpose(1, 2), i32, (3, 2, 32), -1)
    assert binding._rows("x", t(3, 2, 40)[..., :32], i32, (3, 2, 32), -1)[1:] == (80, 40)


def test_rows_below_zero():
    import torch
    t = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ap.AprilError, match="n_rows"):
        ap.april_cache_extend(t(3), t(3), t(3, 4), t(9), t(1), -1)


def test_gradients_are_refused_and_not_silently_left_out():
    import torch
    bf16 = torch.bfloat16
    pool, slots, table, lens = torch.zeros((2, 2, 544), dtype=torch.uint8), torch.zeros(3, dtype=torch.int64), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    x = lambda grad=False: torch.zeros((3, 2, 32), dtype=bf16, requires_grad=grad)  # noqa: E731
    calls = [("q", lambda: ap.april_cache_attention(x(True), pool, table, lens, 60)), ("out", lambda: ap.april_cache_attention(x(), pool, table, lens, 60, out=x(True) * 1)),
             ("lse", lambda: ap.april_cache_attention(x(), pool, table, lens, 60, lse=torch.zeros((3, 2), requires_grad=True))),
             ("k", lambda: ap.april_cache_append(pool, x(True), x(), slots)), ("v", lambda: ap.april_cache_append(pool, x(), x(True) * 2, slots)),
             ("k_values", lambda: ap.april_cache_append(pool, x(), x(), slots, k_values=x(True))), ("v_values", lambda: ap.april_cache_append(pool, x(), x(), slots, v_values=x(True)))]
    for name, call in calls:
        with pytest.raises(ap.AprilError, match="^april error -1: %s requires a gradient" % name):
            call()
        for off in (torch.no_grad, torch.inference_mode):
            with off(), pytest.raises(ap.AprilError, match="not on a GPU"):       # nothing else is wrong with it
                call()


def test_numbers_beyond_their_type_are_refused():
    with pytest.raises(ap.AprilError, match="range"):
        binding._bytes(binding._PACK_EXTEND, 1 << 31, *range(16))


def test_struct_layouts():
    import struct
    for cls, pack, n in ((ap.april_cache_extend_args, "4iq12Q", 17), (ap.april_cache_append_args, "6i4q7Q", 17), (ap.april_cache_attention_args, "9if5q8QqQ", 25)):
        assert C.sizeof(cls) == struct.calcsize(pack) and len(cls._fields_) == n
        values = list(range(3, 3 + n))                          # the packed bytes are the structure's, field by field
        got = cls.from_buffer_copy(struct.pack(pack, *values))
        assert [getattr(got, f) for f, _ in cls._fields_] == values
