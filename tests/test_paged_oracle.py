"""Pins of the paged-cache oracle that need no GPU."""
import numpy as np
import pytest

from oracle import paged_oracle as po


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_rotation_and_depends_on_distance_only(interleaved):
    rng = np.random.default_rng(1)
    f = po.rope_frequencies(32)
    q, k = rng.standard_normal((1, 64)), rng.standard_normal((1, 64))
    a = po.rope(q, [1000], f, interleaved) @ po.rope(k, [993], f, interleaved).T
    b = po.rope(q, [7], f, interleaved) @ po.rope(k, [0], f, interleaved).T
    np.testing.assert_allclose(a, b, rtol=1e-11)
    x = po.rope(q, [123], f, interleaved)
    np.testing.assert_allclose(np.linalg.norm(x), np.linalg.norm(q), rtol=1e-14)
    np.testing.assert_array_equal(x[:, 32:], q[:, 32:])
    np.testing.assert_allclose(po.rope(x, [123], f, interleaved, sign=-1.0), q, atol=1e-13)


def test_the_two_layouts_are_one_map_up_to_the_order_of_the_elements():
    rng = np.random.default_rng(2)
    f, x = po.rope_frequencies(64), rng.standard_normal((3, 64))
    order = np.arange(64).reshape(2, 32).T.ravel()            # halves -> pairs side by side
    np.testing.assert_allclose(po.rope(x, [5, 6, 7], f, False)[:, order], po.rope(x[:, order], [5, 6, 7], f, True), atol=1e-15)


def test_scaling_by_parts_keeps_fast_pairs_and_stretches_slow_ones():
    f = po.rope_frequencies(128, 10000.0)
    s = po.rope_frequencies(128, 10000.0, "by_parts", 4.0, 4096.0)
    turns = 4096 * f / (2 * np.pi)
    np.testing.assert_array_equal(s[turns >= 32], f[turns >= 32])
    np.testing.assert_allclose(s[turns <= 1], f[turns <= 1] / 4, rtol=1e-15)
    assert np.all(np.diff(s) < 0)
    np.testing.assert_allclose(po.rope_frequencies(128, 10000.0, "linear", 8.0), f / 8, rtol=1e-15)


def _pool(rng, B=1, Hkv=2, pages=4, rows=4, D=8):
    table = rng.permutation(B * Hkv * pages).reshape(B, Hkv, pages).astype(np.int32)
    return po.Pool(rng.standard_normal((B * Hkv * pages, rows, D)), rng.standard_normal((B * Hkv * pages, rows, D)), table)


def test_attention_of_a_whole_prompt_is_causal_attention_and_weights_sum_to_the_query_rows():
    import torch
    rng = np.random.default_rng(3)
    pool = _pool(rng)
    n = 13
    Q = rng.standard_normal((1, 4, n, 8))
    end, cnt = np.full((1, 2), n), np.array([n])
    O, lse, w, _, _ = po.attend(Q, pool, end, cnt, True, 8 ** -0.5)
    k, v = (np.stack([np.array([x[pool.at(0, g, j)] for j in range(n)]) for g in range(2)])[None] for x in (pool.K, pool.V))
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(np.repeat(x, r, 1)) for x, r in ((Q, 1), (k, 2), (v, 2))),
                                                            is_causal=True)
    np.testing.assert_allclose(O, want.numpy(), atol=1e-13)
    np.testing.assert_allclose(w.sum(-1), 2 * n, rtol=1e-13)
    assert not w[..., n:].any()


def test_append_then_attend_equals_attend_on_rows_that_were_there():
    rng = np.random.default_rng(4)
    pool = _pool(rng)
    K, V = rng.standard_normal((1, 2, 5, 8)), rng.standard_normal((1, 2, 5, 8))
    row_pos, acc = np.zeros((1, 2, 16), dtype=np.int32), np.ones((1, 2, 16))
    end = po.append(pool, K, V, [40], [5], np.array([[6, 3]]), row_pos, acc)
    np.testing.assert_array_equal(end, [[11, 8]])
    np.testing.assert_array_equal(row_pos[0, 1, 3:8], [40, 41, 42, 43, 44])
    assert not acc[0, 0, 6:11].any() and acc[0, 0, 11] == 1
    np.testing.assert_array_equal(pool.K[pool.at(0, 0, 10)], K[0, 0, 4])
    np.testing.assert_array_equal(pool.V[pool.at(0, 1, 3)], V[0, 1, 0])


def test_eviction_keeps_the_heaviest_rows_and_spares_the_ends():
    rng = np.random.default_rng(5)
    pool = _pool(rng, Hkv=1, pages=4)
    acc = np.array([[[0.1, 5, 5, 0.2, np.nan, 3, 0.0, -0.0, 9, 0.3, 0.3, 1, 0, 0, 0, 0]]])
    pos = np.arange(100, 116, dtype=np.int32)[None, None].copy()
    pos[0, 0, 0] = 0                                       # a sink; the two last of twelve rows are recent
    before = pool.K.copy()
    cnt, pos2, acc2 = po.evict(pool, 6, 1, 2, np.array([112]), np.array([[12]]), pos, acc)
    assert cnt[0, 0] == 6
    # stays: row 0 (sink), 10, 11 (recent), then 9.0, 5.0, 5.0; holes 3, 4, 5 take rows 8, 10, 11
    np.testing.assert_array_equal(pos2[0, 0, :6], [0, 101, 102, 108, 110, 111])
    np.testing.assert_array_equal(acc2[0, 0, :6], [0.1, 5, 5, 9, 0.3, 1])
    np.testing.assert_array_equal(pool.K[pool.at(0, 0, 4)], before[pool.at(0, 0, 10)])
