"""The plain 4-bit cache against its definition by brute force (CPU)."""
import numpy as np
import pytest

from oracle import kv_cache as kc


def test_blocks_take_the_nearest_code_of_the_stated_power():
    rng = np.random.default_rng(0)
    for scale in (1.0, 1e-3, 3e4, 2.0 ** -100):
        for _ in range(50):
            x = (rng.standard_normal(32) * scale).astype(np.float32)
            codes, e = kc.round_block(x)
            y = np.abs(x.astype(np.float64)) / 2.0 ** (e - 127)
            assert 3.5 <= y.max() < 7
            got = kc.open_block(codes, e)
            grid = kc.STEPS * 2.0 ** (e - 127)
            best = np.min(np.abs(np.abs(x.astype(np.float64))[:, None] - grid), axis=1)
            assert np.array_equal(np.abs(np.abs(x.astype(np.float64)) - np.abs(got)), best)
            assert np.all((got == 0) | (np.sign(got) == np.sign(x)))


@pytest.mark.parametrize("top,power", [(1.0, -2), (1.75, -1), (1.7499, -2), (3.5, 0), (7.0, 1), (6.99, 0), (0.0, -125), (2.0 ** -140, -125), (3.4e38, 125)])
def test_power_of_a_block(top, power):
    x = np.zeros(32)
    x[7] = -top
    assert kc.round_block(x)[1] - 127 == power


def test_ties_go_to_the_even_code_and_rounded_values_stay():
    x = np.zeros(32)
    x[:9] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    got = kc.rounded(x)
    assert list(got[:9]) == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -4.0]
    assert np.array_equal(kc.rounded(got), got)
    x[3] = np.inf
    assert np.all(np.isnan(kc.rounded(x)))


def test_rounding_of_many_blocks_is_that_of_each():
    rng = np.random.default_rng(7)
    x = rng.standard_normal((9, 2, 64)) * np.exp2(rng.integers(-140, 128, size=(9, 2, 1)).astype(np.float64))
    x[0, 0, :32] = 0
    x[1, 1, 40] = np.nan
    x[2, 0, :32] = rng.integers(-24, 25, size=32) * 0.25
    each = np.stack([kc.open_block(*kc.round_block(b)) for b in x.reshape(-1, 32)]).reshape(x.shape)
    assert np.array_equal(kc.rounded(x), each, equal_nan=True)


def test_store_and_read():
    rng = np.random.default_rng(1)
    pool = rng.integers(0, 256, size=(5, 2, 17 * 64), dtype=np.uint8)
    before = pool.copy()
    k, v = rng.standard_normal((4, 2, 64)), rng.standard_normal((4, 2, 64))
    slots = [37, -1, 80, 3]                                    # the second and third have no place
    kc.store(pool, k, v, slots)
    got = kc.read(pool, [37, 3])
    assert np.array_equal(got[0], kc.rounded(k[[0, 3]])) and np.array_equal(got[1], kc.rounded(v[[0, 3]]))
    assert np.array_equal(pool[[1, 3, 4]], before[[1, 3, 4]])
    assert np.count_nonzero(pool != before) <= 2 * 2 * 2 * (32 + 2)


def test_tables_over_many_iterations():
    """Every page has one owner at all times, and a token keeps its slot."""
    rng = np.random.default_rng(2)
    n, cols, n_pages = 7, 6, 30
    table, free, lens = [[] for _ in range(n)], list(rng.permutation(n_pages)), [0] * n
    slot_of = {}
    refusals = 0
    for _ in range(200):
        new = [int(rng.integers(-1, 20)) for _ in range(n)]
        held = [-(-x // 16) for x in lens]
        before = ([list(t[:h]) for t, h in zip(table, held)], list(free))
        lens2, starts, slots, pos, status = kc.extend(lens, new, table, free, cols, n_pages, 150)
        if status:
            refusals += 1
            assert [t[:h] for t, h in zip(table, held)] == before[0] and free == before[1] and lens2 == lens and set(slots) == {-1}
            new = [-1 if b == int(rng.integers(n)) else 0 for b in range(n)]
            lens2, starts, slots, pos, status = kc.extend(lens, new, table, free, cols, n_pages, 150)
            assert status == 0
        for b in range(n):
            if new[b] < 0:
                slot_of = {key: s for key, s in slot_of.items() if key[0] != b}
            for r in range(starts[b], starts[b + 1]):
                slot_of[b, pos[r]] = slots[r]
        lens = lens2
        owned = [p for b in range(n) for p in table[b][:-(-lens[b] // 16)]]
        assert sorted(owned + free) == list(range(n_pages))
        assert len(set(slot_of.values())) == len(slot_of) == sum(lens)
        assert all(table[b][p // 16] * 16 + p % 16 == s for (b, p), s in slot_of.items())
    assert refusals > 3


def test_attention_by_brute_force():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 4, 32)), rng.standard_normal((9, 2, 32)), rng.standard_normal((9, 2, 32))
    out, lse, _ = kc.attention(q, k, v, 0.2)
    for i in range(3):
        for h in range(4):
            w = np.array([np.exp(0.2 * sum(q[i, h, d] * k[t, h // 2, d] for d in range(32))) for t in range(7 + i)])
            assert np.allclose(out[i, h], (w[:, None] * v[:7 + i, h // 2]).sum(0) / w.sum()) and np.isclose(lse[i, h], np.log(w.sum()))
    out, lse, _ = kc.attention(q, k[:1], v[:1], 0.2)           # the first two rows see nothing
    assert np.all(out[:2] == 0) and np.all(lse[:2] == -np.inf) and np.allclose(out[2], v[0].repeat(2, axis=0))
