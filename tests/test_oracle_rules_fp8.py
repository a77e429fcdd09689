"""Pins of the oracle's sampling rules and 8-bit rounding (no GPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import fp8, rules, sampling


def test_e4m3_rounding_equals_torchs_cast():
    """Every e4m3 value, every midpoint, and values around them (float32 in both)."""
    t = fp8.e4m3_values()
    assert t[-1] == 448 and t[1] == 2.0 ** -9
    mid = (t[1:] + t[:-1]) / 2
    x = np.concatenate([t, mid, np.nextafter(mid.astype(np.float32), np.float32(1e9)),
                        np.nextafter(mid.astype(np.float32), np.float32(0)),
                        np.random.default_rng(0).normal(0, 60, 4000).clip(-448, 448)]).astype(np.float32)
    x = np.concatenate([x, -x])
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(fp8.round_e4m3(x), ref)
    assert np.isnan(fp8.round_e4m3(np.array([np.nan, np.inf, -np.inf]))).all()


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.5, 1), (449.0, 1), (224.0, -1), (1.75, -8), (1.7578125, -7),
                                    (0.0, -100), (2.0 ** -130, -100)])
def test_block_scale(amax, e):
    x = np.zeros((64, 8))
    x[3, 5] = -amax
    assert fp8.block_scale(x) == 2.0 ** e
    x[7, 1] = np.inf
    x[8, 1] = np.nan
    assert fp8.block_scale(x) == 2.0 ** e  # (the finite entries decide)


def test_stored_error_is_within_half_a_step():
    """|stored - x| <= 2^-4 |x| + half the smallest subnormal's step, and rows past the sealed ones are untouched."""
    x = np.random.default_rng(1).normal(0, 1.3, (130, 2, 32))
    y = fp8.stored(x, 128)
    s = np.stack([[fp8.block_scale(x[p:p + 64, g]) for g in range(2)] for p in (0, 64)]).repeat(64, 0)[:, :, None]
    assert (np.abs(y[:128] - x[:128]) <= np.abs(x[:128]) * 2.0 ** -4 + s * 2.0 ** -10).all()
    np.testing.assert_array_equal(y[128:], x[128:])


def test_attention_equals_torchs():
    r = np.random.default_rng(2)
    q, k, v = r.normal(size=(3, 4, 16)), r.normal(size=(9, 2, 16)), r.normal(size=(9, 2, 16))
    o = fp8.attention(q, k, v, 6)
    t = lambda x: torch.from_numpy(x).transpose(0, 1)  # noqa: E731
    mask = torch.arange(9)[None] <= 6 + torch.arange(3)[:, None]
    ref = torch.nn.functional.scaled_dot_product_attention(t(q), t(k).repeat_interleave(2, 0),
                                                           t(v).repeat_interleave(2, 0), attn_mask=mask)
    np.testing.assert_allclose(o, ref.transpose(0, 1).numpy(), atol=1e-12)


def test_rules_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3])).astype(np.float32)
    order = lambda **kw: list(rules.kept(l, **kw)[0])  # noqa: E731
    assert order() == [1, 3, 2, 0]
    assert order(top_k=2) == [1, 3]
    assert order(top_p=0.39) == [1] and order(top_p=0.41) == [1, 3] and order(top_p=0.0) == [1]
    assert order(min_p=0.6) == [1, 3] and order(min_p=1.0) == [1] and order(min_p=7.0) == [1]
    # top-p counts the mass of the top-k: 0.4 / 0.7 = 0.571
    assert order(top_k=2, top_p=0.57) == [1] and order(top_k=2, top_p=0.58) == [1, 3]
    assert order(T=0.0) == [1]
    p = rules.probabilities(l, top_k=2)
    np.testing.assert_allclose(p, [0, 4 / 7, 0, 3 / 7], rtol=1e-6)


def test_rules_ties_and_masks():
    l = np.array([1.0, 3.0, 3.0, -np.inf, 3.0, 1.0], np.float32)
    assert list(rules.kept(l, top_k=2)[0]) == [1, 2]  # equal logits: the lower index first
    assert list(rules.kept(l, top_k=4)[0]) == [1, 2, 4, 0]
    assert list(rules.kept(l, top_k=99)[0]) == [1, 2, 4, 0, 5]
    assert rules.probabilities(l)[3] == 0
    for bad in ([np.nan, 1.0], [np.inf, 1.0], [-np.inf, -np.inf]):
        with pytest.raises(sampling.NonFiniteError):
            rules.kept(np.array(bad))
    for rule in ({"T": -1.0}, {"T": math.nan}, {"top_p": math.nan}, {"min_p": math.nan}):
        with pytest.raises(sampling.NonFiniteError):
            rules.kept(l, **rule)


def test_rules_off_is_the_softmax():
    l = np.random.default_rng(3).normal(0, 2, 500)
    np.testing.assert_allclose(rules.probabilities(l, T=0.7), sampling.softmax(l, 0.7), rtol=2.0 ** -23)


def test_truncated_rows_keep_the_output_distribution():
    """Accept / resample on truncated p and q draws from the truncated p: over
    all accept words (here the exact probabilities) P(token) = p."""
    r = np.random.default_rng(4)
    p = rules.probabilities(r.normal(0, 1, 6), top_k=4).astype(np.float64)
    q = rules.probabilities(r.normal(0, 1, 6), top_p=0.8).astype(np.float64)
    acc = np.minimum(p, q)
    resid = np.maximum(p - q, 0)
    out = acc + (1 - acc.sum()) * resid / resid.sum()
    np.testing.assert_allclose(out, p / p.sum(), atol=3e-7)
