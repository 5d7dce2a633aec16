"""Pins of the oracle of the paged-cache operators: closed forms and a slow second way of writing each."""
import math

import numpy as np
import pytest

from oracle import paged_kv as O


def _rand(*shape, seed=0):
    return np.random.default_rng(seed).standard_normal(shape)


def test_without_window_it_is_the_decoders_causal_attention():
    import torch
    q, k, v = _rand(5, 6, 8, seed=1), _rand(9, 2, 8, seed=2), _rand(9, 2, 8, seed=3)
    out, lse, p, mag, big = O.attention(q, k, v, 8 ** -0.5)
    tq = torch.from_numpy(q).transpose(0, 1)
    tk, tv = (torch.from_numpy(x).repeat_interleave(3, dim=1).transpose(0, 1) for x in (k, v))
    mask = torch.ones(5, 9, dtype=torch.bool).tril(4)
    ref = torch.nn.functional.scaled_dot_product_attention(tq[None], tk[None], tv[None], attn_mask=mask)[0]
    np.testing.assert_allclose(out, ref.transpose(0, 1).numpy(), atol=1e-12)
    np.testing.assert_allclose(p.sum(axis=2), 1.0, atol=1e-12)
    assert np.all(mag >= np.abs(out) - 1e-12) and np.all(big > 0)


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (4, 0), (100, 3), (2, 100)])
def test_window_and_sinks_row_by_row(window, sinks):
    T, n = 11, 7
    q, k, v = _rand(n, 2, 4, seed=4), _rand(T, 1, 4, seed=5), _rand(T, 1, 4, seed=6)
    out, lse, p, _, _ = O.attention(q, k, v, 0.7, window, sinks)
    for i in range(n):
        t = T - n + i
        js = [j for j in range(t + 1) if j < sinks or j > t - window]
        for h in range(2):
            e = [math.exp(0.7 * float(q[i, h] @ k[j, 0])) for j in js]
            np.testing.assert_allclose(out[i, h], sum(w * v[j, 0] for w, j in zip(e, js)) / sum(e), atol=1e-12)
            assert abs(lse[i, h] - math.log(sum(e))) < 1e-12
            assert [j for j in range(T) if p[i, h, j] > 0] == js


def test_rows_that_see_nothing_and_absent_tokens():
    q, k, v = _rand(4, 2, 4), _rand(2, 1, 4), _rand(2, 1, 4)
    out, lse, p, _, _ = O.attention(q, k, v, 1.0)               # rows 0 and 1 sit below slot 0
    assert np.all(out[:2] == 0) and np.all(np.isneginf(lse[:2])) and np.all(np.isfinite(lse[2:]))
    k[0], v[0] = np.nan, np.inf
    out, lse, p, _, _ = O.attention(q[2:], k, v, 1.0, there=[False, True])
    assert np.all(out[0] == 0) and np.all(np.isneginf(lse[0]))
    np.testing.assert_allclose(out[1, 0], v[1, 0])


def test_score_is_the_derivative_of_the_summed_lse():
    """d lse_ih / d (scale q_ih . k_j) = p_ij: nudging every score with token j of a KV head gives its weight."""
    q, k, v = _rand(3, 4, 6, seed=7), _rand(8, 2, 6, seed=8), _rand(8, 2, 6, seed=9)
    _, _, p, _, _ = O.attention(q, k, v, 0.5, 4, 1)
    w = O.score(p, 2)
    np.testing.assert_allclose(w.sum(), 3 * 4, atol=1e-12)
    extra = np.concatenate([q, np.ones((3, 4, 1))], axis=2)
    for g in range(2):
        for j in range(8):
            total = []
            for step in (1e-5, -1e-5):
                nudge = np.zeros((8, 2, 1))
                nudge[j, g] = step / 0.5
                lse = O.attention(extra, np.concatenate([k, nudge], axis=2), np.zeros((8, 2, 7)), 0.5, 4, 1)[1]
                total.append(lse.sum())
            assert abs((total[0] - total[1]) / 2e-5 - w[g, j]) < 1e-8


def test_evict_against_a_selection_one_by_one():
    rng = np.random.default_rng(3)
    for _ in range(50):
        T = int(rng.integers(1, 30))
        s = np.round(rng.random(T) * 4) / 4                       # many ties
        s[rng.random(T) < 0.1] = np.nan
        sinks, recent = int(rng.integers(0, 5)), int(rng.integers(0, 5))
        budget = max(1, sinks + recent + int(rng.integers(0, 12)))
        kept = O.evict(s, budget, sinks, recent)
        if T <= budget:
            assert kept == list(range(T))
            continue
        left = list(range(sinks, T - recent))
        want = list(range(sinks)) + list(range(T - recent, T))
        for _ in range(budget - sinks - recent):
            j = left[0]
            for x in left:
                if (np.isnan(s[j]) and not np.isnan(s[x])) or s[x] > s[j]:
                    j = x
            left.remove(j)
            want.append(j)
        assert kept == sorted(want) and len(kept) == budget
