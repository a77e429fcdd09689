"""The oracle's norm and rotation against closed forms (no GPU needed)."""
import numpy as np
import pytest
import torch

from oracle import model, rope


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rot", [(32, 32), (64, 16), (128, 128), (64, 0)])
def test_a_pair_is_a_complex_number_turned(hd, rot, interleaved):
    rng = np.random.default_rng(hd + rot)
    x, pos = rng.normal(size=(2, 3, 4, hd)), rng.integers(0, 10000, (2, 3))
    f = rope.freqs(rot, 10000.0)
    y = rope.apply(x, pos, f, interleaved)
    a, b = rope.pairs(rot, interleaved)
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, :, None, None] * f)
    np.testing.assert_allclose(y[..., a] + 1j * y[..., b], z, atol=1e-12)
    np.testing.assert_array_equal(y[..., rot:], x[..., rot:])
    np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 1, 1, 1, 64))
    f = rope.freqs(64, 10000.0)
    dot = lambda i, j: (rope.apply(q, [[i]], f) * rope.apply(k, [[j]], f)).sum()  # noqa: E731
    np.testing.assert_allclose(dot(1234, 1000), dot(234, 0), atol=1e-10)


def test_norm_and_the_decoders_rotation():
    rng = np.random.default_rng(2)
    x, g = rng.normal(size=(1, 3, 2, 64)), rng.normal(size=64)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(g), 1e-5).numpy()
    np.testing.assert_allclose(rope.norm(x, g, 1e-5), ref, atol=1e-12)
    pos = np.array([[5, 6, 7]])
    np.testing.assert_allclose(rope.apply(x, pos, rope.freqs(64, 10000.0))[0], model.rope(x[0], pos[0], 10000.0),
                               atol=1e-12)
