"""Pins of the scored-attention oracle: closed forms, library special cases, the
keyless oracle as the case without cap, bias or mask, finite differences."""

import numpy as np
import pytest
import torch

from oracle import keyless as K
from oracle import scored as S


def _rand(seed, *shape):
    return np.random.RandomState(seed).standard_normal(shape)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,G", [(4, 4), (4, 2), (4, 1)])
def test_plain_scores_are_the_keyless_attention(causal, H, G):
    q, v, g = _rand(1, 2, 9, H, 8), _rand(2, 2, 9, G, 8), _rand(3, 2, 9, H, 8)
    seen = S.row_ranges(2, 9, causal=causal)
    out, lse = S.scored_attention(q, v, seen=seen)
    np.testing.assert_allclose(lse, K.attention_logsumexp(q, v, H, G, 8, causal), atol=1e-12)
    for i in range(9):
        n = i + 1 if causal else 9
        np.testing.assert_allclose(out[1, i, 3], K.decode_one(q[1, i, 3], v[1, :n, 3 // (H // G)]), atol=1e-12)
    for a, b in zip(S.scored_attention_backward(q, v, g, seen=seen),
                    K.keyless_attention_backward(q, v, g, H, G, 8, causal)):
        np.testing.assert_allclose(a, b, atol=1e-12)


def test_bias_and_documents_are_an_additive_mask():
    """Against torch's attention with keys := values and an additive mask."""
    B, N, H, G, d = 2, 11, 4, 2, 8
    q, v = _rand(4, B, N, H, d), _rand(5, B, N, G, d)
    slopes = np.array([0.5, 0.25, -0.125, 1.0])
    first = np.array([[0] * 4 + [4] * 7, [0] * 9 + [9] * 2])
    last = np.maximum(np.arange(N) + 1, first + 2)
    out, _ = S.scored_attention(q, v, slopes=slopes, seen=S.row_ranges(B, N, first, last))
    i = np.arange(N)
    bias = -slopes[None, :, None, None] * np.abs(i[:, None] - i[None])
    ok = (i >= first[:, :, None]) & (i < last[:, :, None])
    bias = np.where(ok[:, None], bias, -np.inf)
    t = torch.from_numpy
    kv = t(np.repeat(v, H // G, 2)).permute(0, 2, 1, 3)
    ref = torch.nn.functional.scaled_dot_product_attention(t(q).permute(0, 2, 1, 3), kv, kv, t(bias))
    np.testing.assert_allclose(out, ref.permute(0, 2, 1, 3).numpy(), atol=1e-12)


def test_capped_scores_closed_form():
    """One query, two values: z = (large, 0), so the scores are (cap tanh, 0)."""
    q, v = np.zeros((1, 2, 1, 4)), np.zeros((1, 2, 1, 4))
    q[0, 1, 0, 0], v[0, 0, 0, 0] = 10.0, 3.0
    out, lse = S.scored_attention(q, v, cap=2.0, seen=S.row_ranges(1, 2), scale=1.0)
    e = np.exp(2.0 * np.tanh(15.0))
    assert out[0, 1, 0, 0] == pytest.approx(3.0 * e / (e + 1.0))
    assert lse[0, 0, 1] == pytest.approx(np.log(e + 1.0))
    # A cap far above the scores changes nothing to first order.
    a = S.scored_attention(q, v, cap=1e6, seen=S.row_ranges(1, 2), scale=0.01)[0]
    np.testing.assert_allclose(a, S.scored_attention(q, v, seen=S.row_ranges(1, 2), scale=0.01)[0], atol=1e-9)


def test_rows_that_see_nothing():
    q, v, g = _rand(6, 1, 5, 2, 4), _rand(7, 1, 5, 1, 4), _rand(8, 1, 5, 2, 4)
    last = np.array([[0, 2, 3, 4, 5]])
    seen = S.row_ranges(1, 5, None, last)
    out, lse = S.scored_attention(q, v, 3.0, seen=seen)
    assert (out[0, 0] == 0).all() and (lse[0, :, 0] == -np.inf).all()
    dq, dv = S.scored_attention_backward(q, v, g, 3.0, seen=seen)
    assert (dq[0, 0] == 0).all()
    g2 = g.copy()
    g2[0, 0] = 100.0
    np.testing.assert_array_equal(S.scored_attention_backward(q, v, g2, 3.0, seen=seen)[1], dv)


@pytest.mark.parametrize("cap", [0.0, 1.5])
def test_gradients_by_central_differences(cap):
    B, N, H, G, d = 1, 6, 4, 2, 4
    q, v, g = _rand(9, B, N, H, d), _rand(10, B, N, G, d), _rand(11, B, N, H, d)
    slopes = np.array([0.3, 0.0, -0.2, 0.7])
    first = np.array([[0, 0, 0, 3, 3, 3]])
    last = np.array([[2, 2, 3, 4, 6, 6]])
    seen = S.row_ranges(B, N, first, last)

    def loss(q, v):
        return float((S.scored_attention(q, v, cap, slopes, seen)[0] * g).sum())
    dq, dv = S.scored_attention_backward(q, v, g, cap, slopes, seen)
    h = 1e-5
    for x, grad, at in ((q, dq, lambda x: loss(x, v)), (v, dv, lambda x: loss(q, x))):
        for k in np.random.RandomState(12).choice(x.size, 20, replace=False):
            up, down = x.copy(), x.copy()
            up.flat[k] += h
            down.flat[k] -= h
            assert (at(up) - at(down)) / (2 * h) == pytest.approx(grad.flat[k], rel=1e-6, abs=1e-8)


def test_chain_and_paths_of_a_tree_are_prefills():
    """A chain over a cache equals the last rows of the causal attention; each path of
    a tree equals the chain of its tokens."""
    n, T, H, G, d, cap = 7, 5, 4, 2, 8, 2.0
    slopes = np.array([0.5, 0.1, 0.0, -0.3])
    v, q = _rand(13, 1, n + T, G, d), _rand(14, 1, n + T, H, d)
    cache = v.transpose(0, 2, 1, 3)
    full, _ = S.scored_attention(q, v, cap, slopes, S.row_ranges(1, n + T))
    chain = S.tree_decode(q[:, n:], cache, [n], None, H, G, cap, slopes)
    np.testing.assert_allclose(chain, full[:, n:], atol=1e-12)
    words = S.tree_words([[-1, 0, 0, 1, 2]])
    assert [int(w) for w in words[0]] == [1, 3, 5, 11, 21]
    got = S.tree_decode(q[:, n:], cache, [n], words, H, G, cap, slopes)
    for path in ([0, 1, 3], [0, 2, 4]):
        rows = np.concatenate([v[:, :n], v[:, n:][:, path]], 1).transpose(0, 2, 1, 3)
        one = S.tree_decode(q[:, n:][:, path], rows, [n], None, H, G, cap, slopes)
        np.testing.assert_allclose(got[:, path], one, atol=1e-12)


def test_keep_then_decode_is_the_accepted_chain():
    cache = _rand(15, 2, 3, 12, 4)
    path, kept = np.array([[1, 3, 0], [0, 0, 0]]), np.array([2, 0])
    new = S.value_cache_keep(cache, [5, 8], path, kept)
    np.testing.assert_array_equal(new[0, :, 5], cache[0, :, 6])
    np.testing.assert_array_equal(new[0, :, 6], cache[0, :, 8])
    same = np.ones((2, 3, 12), bool)
    same[0, :, 5:7] = False
    np.testing.assert_array_equal(new[same], cache[same])
    # Paged, in shuffled blocks: the same rows by position.
    table = np.array([[2, 0, 3], [5, 4, 1]])
    paged = np.zeros((6, 3, 4, 4))
    for b in range(2):
        for i in range(12):
            paged[table[b][i // 4], :, i % 4] = cache[b, :, i]
    moved = S.value_cache_keep(paged, [5, 8], path, kept, table, 4)
    for b in range(2):
        for g in range(3):
            np.testing.assert_array_equal(K.cache_rows(moved, b, g, 12, table, 4), new[b, g])
