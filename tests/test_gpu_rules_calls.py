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
