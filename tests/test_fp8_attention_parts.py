"""That the bound of tests/fp8_parts.py tells the parts that attention's products
take from fewer: an emulation in float32 with all of them is within it, one
with a part less, of the queries or of the probabilities, is not."""
import numpy as np
import pytest

from tests import fp8_parts


def _bf16(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32)


def _fp16(x):
    return np.asarray(x, np.float32).astype(np.float16).astype(np.float32)


def _parts(x, rnd, count):
    out, rest = [], np.asarray(x, np.float32)
    for _ in range(count):
        out.append(rnd(rest))
        rest = rest - out[-1]  # (exact)
    return out[::-1]  # small ones first


def _emulate(q, k, rnd, q_parts, p_parts, lift):
    """float32 attention of the two keys, queries (those of fp16 brought to 2^13) and probabilities in parts."""
    f = np.float32
    hd = q.shape[-1]
    v = q * f(f(1.44269504) / np.sqrt(f(hd)))
    shift = np.exp2(13 - np.floor(np.log2(np.abs(v).max(-1, keepdims=True)))).astype(f) if rnd is _fp16 else f(1)
    s = []
    for key in (fp8_parts.A, fp8_parts.B):
        acc = np.zeros(q.shape[:-1], f)
        for part in _parts(v * shift, rnd, q_parts):
            acc = acc + (part * k[key].astype(f)).sum(-1, dtype=f)  # (one term is not zero)
        s.append(acc * (f(1) / np.broadcast_to(shift, v.shape)[..., 0]))
    m = np.maximum(*s)
    p = [np.exp2(x.astype(np.float64) + (f(lift) - m)).astype(f) for x in s]
    num = np.zeros_like(m)
    for part in _parts(p[1], rnd, p_parts):
        num = num + part
    return num / (p[0] + p[1])


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("kind", ["scores", "probabilities"])
@pytest.mark.parametrize("n,H", [(1, 64), (70, 2)])
def test_the_bound_tells_the_parts(kind, hd, n, H):
    q, k, v, s1, s2 = fp8_parts.inputs(kind, hd, H, n, 128, seed=hd + n)
    ref, tol = fp8_parts.reference(s1, s2), fp8_parts.bound(s1, s2)
    worst = lambda *a: (np.abs(_emulate(q, k, *a) - ref) / tol).max()  # noqa: E731
    assert worst(_bf16, 3, 3, 0) < 0.75 and worst(_fp16, 2, 2, 15) < 0.75
    fewer_bf16 = worst(_bf16, 2, 3, 0) if kind == "scores" else worst(_bf16, 3, 2, 0)
    fewer_fp16 = worst(_fp16, 1, 2, 15) if kind == "scores" else worst(_fp16, 2, 1, 15)
    print(kind, hd, n, worst(_bf16, 3, 3, 0), worst(_fp16, 2, 2, 15), fewer_bf16, fewer_fp16)
    assert fewer_bf16 > 1.5 and fewer_fp16 > 30


def test_what_parts_leave():
    """Three bf16 parts hold a float32 whole, two leave at most 2^-17, two of fp16 2^-23."""
    x = np.random.default_rng(1).uniform(1, 2, 200000).astype(np.float32)
    x[:3] = np.nextafter(np.float32(2), np.float32(1)), 1 + 2.0 ** -8, 1 + 2.0 ** -8 - 2.0 ** -23
    left = lambda rnd, n: np.abs(x - sum(_parts(x, rnd, n)[::-1], np.zeros_like(x, np.float64))).max()  # noqa: E731
    assert left(_bf16, 3) == 0
    assert 2.0 ** -18 < left(_bf16, 2) <= 2.0 ** -17 and left(_bf16, 1) <= 2.0 ** -8
    assert left(_fp16, 2) <= 2.0 ** -23 and left(_fp16, 1) <= 2.0 ** -11
