"""Calls of specdec_sample_logits that its documentation allows, beside those of tests/test_gpu_rules.py."""
import numpy as np
import pytest

from oracle import rules
from oracle.sampling import sample_fixed_point
from paper_2608_10362_amd import binding, synth
from tests.gpu_util import f32, i32, log, torch_cuda, u32_tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,R,V", [(3, 1, 1000), (2, 3, 4099)])
def test_logits_and_probabilities_alternate_in_one_buffer(B, R, V):
    """Rows of one stride that lie between each other's do not overlap."""
    torch = torch_cuda()
    rng = np.random.default_rng(V)
    logits, words = rng.normal(0, 2, (B, R, V)).astype(np.float32), synth.make_rand_u32((B, R), seed=V)
    sr = binding.SamplingRules(top_k=i32([9] * B), top_p=f32([0.8] * B))
    log(f"alternating rows {B} x {R} x {V}")
    for first in (0, 1):  # (logits before the probabilities, and after)
        both = torch.full((B, R, 2, V), -5.0, device="cuda")
        both[:, :, first] = f32(logits)
        out = torch.zeros((B, R), dtype=torch.int32, device="cuda")
        binding.specdec_sample_logits(both[:, :, first], sr, rand=u32_tensor(words), probs=both[:, :, 1 - first], out=out)
        np.testing.assert_array_equal(both[:, :, first].cpu().numpy(), logits)
        p = both[:, :, 1 - first].cpu().numpy()
        for b in range(B):
            for i in range(R):
                ref = rules.probabilities(logits[b, i], top_k=9, top_p=float(np.float32(0.8)))
                np.testing.assert_allclose(p[b, i], ref, rtol=2.0 ** -22)
                assert int(out[b, i]) == sample_fixed_point(ref, int(words[b, i]))


def _checked(logits, r, p, tok, word):
    ref = rules.probabilities(logits, **r)
    np.testing.assert_array_equal(p > 0, ref > 0)
    np.testing.assert_allclose(p, ref, rtol=2.0 ** -22, atol=2.0 ** -140)
    assert int(tok) == sample_fixed_point(ref, int(word))


@pytest.mark.parametrize("B,R", [(128, 5), (1600, 1)])
def test_a_long_top_k_over_many_rows(B, R):
    """So many rows have few workgroups each, and fewer group maxima than a long top-k:
    such a row's candidates are all its entries, more than a list holds."""
    torch = torch_cuda()
    V, rng = 8000, np.random.default_rng(B)
    logits, words = rng.normal(0, 2.5, (B, R, V)).astype(np.float32), synth.make_rand_u32((B, R), seed=B)
    kinds = [{"top_k": 1000, "T": 0.7}, {"top_k": 253, "top_p": 0.9}, {"top_k": 3000}, {"top_k": 50, "T": 1.5}]
    each = [kinds[b % 4] for b in range(B)]
    sr = binding.SamplingRules(temperature=f32([r.get("T", 1.0) for r in each]), top_k=i32([r["top_k"] for r in each]),
                               top_p=f32([r.get("top_p", 1.0) for r in each]))
    lg, wd = f32(logits), u32_tensor(words)
    probs, out = torch.full_like(lg, float("nan")), torch.full((B, R), -7, dtype=torch.int32, device="cuda")
    log(f"long top-k over {B} x {R} rows")
    binding.specdec_sample_logits(lg, sr, rand=wd, probs=probs, out=out)
    p, tok = probs.cpu().numpy(), out.cpu().numpy()
    for b in list(range(8)) + list(range(B - 8, B)):
        r = {k: (x if k == "top_k" else float(np.float32(x))) for k, x in each[b].items()}
        for i in range(R):
            _checked(logits[b, i], r, p[b, i], tok[b, i], words[b, i])
    alone = torch.full_like(out, -7)
    binding.specdec_sample_logits(lg, sr, rand=wd, out=alone)
    assert torch.equal(alone, out)


def test_the_largest_sizes():
    """65535 rows in one call; a vocabulary of 2^20."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    B, R, V = 21845, 3, 40
    logits, words = rng.normal(0, 2, (B, R, V)).astype(np.float32), synth.make_rand_u32((B, R), seed=3)
    k = (np.arange(B) % 7).astype(np.int32)
    sr = binding.SamplingRules(top_k=i32(k), top_p=f32([0.9] * B))
    lg = f32(logits)
    probs, out = torch.full_like(lg, float("nan")), torch.full((B, R), -7, dtype=torch.int32, device="cuda")
    log("65535 rows")
    binding.specdec_sample_logits(lg, sr, rand=u32_tensor(words), probs=probs, out=out)
    p, tok = probs.cpu().numpy(), out.cpu().numpy()
    assert np.isfinite(p).all() and (tok >= 0).all()
    for b in [0, 1, 2, 3, 4, 5, 6, 10000, B - 2, B - 1]:
        for i in range(R):
            _checked(logits[b, i], {"top_k": int(k[b]), "top_p": float(np.float32(0.9))}, p[b, i], tok[b, i], words[b, i])
    V, names = 2 ** 20, [{}, {"top_k": 700}, {"top_p": 0.95}, {"min_p": 0.01, "T": 1.3}]
    logits, words = rng.normal(0, 2, (len(names), V)).astype(np.float32), synth.make_rand_u32(len(names), seed=4)
    words[0] = 0xFFFFFFFF
    sr = binding.SamplingRules(temperature=f32([r.get("T", 1.0) for r in names]), top_k=i32([r.get("top_k", 0) for r in names]),
                               top_p=f32([r.get("top_p", 1.0) for r in names]), min_p=f32([r.get("min_p", 0.0) for r in names]))
    lg = f32(logits)
    probs, out = torch.full_like(lg, float("nan")), torch.full((len(names),), -7, dtype=torch.int32, device="cuda")
    log("a vocabulary of 2^20")
    binding.specdec_sample_logits(lg, sr, rand=u32_tensor(words), probs=probs, out=out)
    for b, r in enumerate(names):
        r = {n: (x if n == "top_k" else float(np.float32(x))) for n, x in r.items()}
        _checked(logits[b], r, probs[b].cpu().numpy(), out[b], words[b])


def test_two_calls_at_once_and_rules_that_change_between_replays():
    """Calls on two streams, each with a workspace; a captured call reads the rules' values at each replay."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    B, V, sets = 6, 30000, 4
    logits = [rng.normal(0, 2.5, (B, V)).astype(np.float32) for _ in range(2)]
    words = [synth.make_rand_u32(B, seed=6 + j) for j in range(2)]
    T, K, P = (f32([1.0] * B), i32([0] * B), f32([1.0] * B))
    sr = binding.SamplingRules(temperature=T, top_k=K, top_p=P)
    lg, wd = [f32(x) for x in logits], [u32_tensor(x) for x in words]
    outs = [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)]
    probs = [torch.empty_like(lg[0]) for _ in range(2)]
    ws = [binding.sample_workspace(B, 1, V) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[j]):
            binding.specdec_sample_logits(lg[j], sr, rand=wd[j], probs=probs[j], out=outs[j], workspace=ws[j])
        graphs.append(g)
    for i in range(sets):
        k = [[0, 50, 1, 2000, 0, 9], [40] * B, [0] * B, [0, 0, 3, 400, 64, 1000]][i]
        p = [[1.0, 0.9, 0.5, 0.99, 0.7, 1.0], [1.0] * B, [0.8] * B, [1.0, 0.3, 1.0, 0.9, 1.0, 1.0]][i]
        t = [[1.0] * B, [0.0, 0.5, 1.0, 2.0, 0.0, 1.0], [0.7] * B, [1.5] * B][i]
        K.copy_(i32(k)); P.copy_(f32(p)); T.copy_(f32(t))
        torch.cuda.synchronize()
        log(f"two graphs at once, rules {i}")
        for rep in range(3):
            for j in range(2):
                with torch.cuda.stream(streams[j]):
                    graphs[j].replay()
        torch.cuda.synchronize()
        eager = [(x.cpu().numpy().copy(), o.cpu().numpy().copy()) for x, o in zip(probs, outs)]
        for j in range(2):
            for b in range(B):
                r = {"T": float(np.float32(t[b])), "top_k": k[b], "top_p": float(np.float32(p[b]))}
                _checked(logits[j][b], r, eager[j][0][b], eager[j][1][b], words[j][b])
        for j in range(2):  # eager calls on both streams, one after the other without a wait
            binding.specdec_sample_logits(lg[j], sr, rand=wd[j], probs=probs[j], out=outs[j], workspace=ws[j], stream=streams[j])
        torch.cuda.synchronize()
        for j in range(2):
            np.testing.assert_array_equal(probs[j].cpu().numpy(), eager[j][0])
            np.testing.assert_array_equal(outs[j].cpu().numpy(), eager[j][1])
