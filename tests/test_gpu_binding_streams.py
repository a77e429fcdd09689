"""Calls on a stream other than the current one, with workspaces of their own:
right results, and memory that the current stream is not given while the call
may still use it (the allocations themselves: tests/test_binding_streams.py)."""
import numpy as np
import pytest

from oracle import fp8, rules
from oracle.sampling import sample_fixed_point
from paper_2608_10362_amd import binding, synth
from tests.gpu_util import f32, i32, log, torch_cuda, u32_tensor

pytestmark = pytest.mark.gpu


def _watched(monkeypatch, name):
    """The (address, bytes) of every workspace that binding.<name> hands out."""
    seen, make = [], getattr(binding, name)

    def watch(*args):
        t = make(*args)
        seen.append((t.data_ptr(), t.numel()))
        return t
    monkeypatch.setattr(binding, name, watch)
    return seen


def _not_handed_out(seen, side):
    """The workspace's memory stays with the side stream."""
    torch = torch_cuda()
    (at, n), = seen
    here = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert at not in [t.data_ptr() for t in here]
    with torch.cuda.stream(side):
        there = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert there.data_ptr() == at


def test_attention(monkeypatch):
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    L, n, H, G, hd = 4000, 1, 4, 1, 64  # (parts of one unit: the workspace is written)
    shape = synth.ModelShape(1, H * hd, H, G, hd, 128, 64)
    kv = binding.Fp8KVCache(shape, 1, 4096, 128)
    k, v = (torch.from_numpy(rng.normal(0, 1, (L + n, G, hd)).astype(np.float32)).cuda().bfloat16() for _ in range(2))
    kv.write_context(0, 0, 0, k[:L].contiguous(), v[:L].contiguous())
    kv.set_state([L], [[0, 1]], [1])
    binding.specdec_kv_append(kv, 0, k[None, L:].contiguous(), v[None, L:].contiguous())
    q = torch.from_numpy(rng.normal(0, 1, (1, n, H, hd)).astype(np.float32)).cuda()
    want, got = torch.empty_like(q), torch.empty_like(q)
    binding.specdec_attention(kv, 0, q, want)
    torch.cuda.synchronize()
    side, seen = torch.cuda.Stream(), _watched(monkeypatch, "attention_workspace")
    log("attention on a side stream")
    binding.specdec_attention(kv, 0, q, got, stream=side)
    _not_handed_out(seen, side)
    side.synchronize()
    torch.testing.assert_close(got, want, rtol=0, atol=0)
    # rows read back on the side stream, used and dropped on the current one
    a, b = kv.read_context(0, 0, 0, L, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    a, b = a.float().cpu().numpy(), b.float().cpu().numpy()
    for x, ref in ((a, k), (b, v)):
        np.testing.assert_array_equal(x, fp8.stored(ref[:L].float().cpu().numpy(), L // 64 * 64))


def test_sample_logits_and_accept(monkeypatch):
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    B, V = 3, 20000
    logits, words = rng.normal(0, 2.5, (B, V)).astype(np.float32), synth.make_rand_u32(B, seed=4)
    sr = binding.SamplingRules(top_k=i32([40, 0, 2000]), top_p=f32([0.9, 0.8, 1.0]))
    lg, wd = f32(logits), u32_tensor(words)
    out = torch.zeros(B, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    side, seen = torch.cuda.Stream(), _watched(monkeypatch, "sample_workspace")
    log("sampling on a side stream")
    binding.specdec_sample_logits(lg, sr, rand=wd, out=out, stream=side)
    _not_handed_out(seen, side)
    side.synchronize()
    for b, r in enumerate(({"top_k": 40, "top_p": float(np.float32(0.9))}, {"top_p": float(np.float32(0.8))},
                           {"top_k": 2000})):
        assert int(out[b]) == sample_fixed_point(rules.probabilities(logits[b], **r), int(words[b]))

    seen = _watched(monkeypatch, "accept_workspace")
    d = i32(logits.argmax(1).reshape(B, 1))
    p = f32(np.stack([logits, logits], 1))
    n_acc, nxt = (torch.full((B,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    log("accept on a side stream")
    binding.specdec_accept(B, 1, V, binding.INPUT_LOGITS, 0.0, p, None, d, 1, None, 0, 0, n_acc, nxt, stream=side)
    _not_handed_out(seen, side)
    side.synchronize()
    assert n_acc.tolist() == [1] * B and nxt.tolist() == logits.argmax(1).tolist()
