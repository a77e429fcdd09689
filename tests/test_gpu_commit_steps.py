"""What a commit adds to the lengths is what it seals in an 8-bit cache: lengths against
the rule of both roles, and the blocks that were completed rounded, for every accepted count."""
import numpy as np
import pytest

from oracle import fp8
from paper_2608_10362_amd import binding
from tests.gpu_util import i32, log, torch_cuda
from tests.test_gpu_fp8_cache import _bf16, _cache, _np, _rows, _shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("role", [binding.ROLE_TARGET, binding.ROLE_DRAFT], ids=["target", "draft"])
@pytest.mark.parametrize("n_pending", [1, 2])
def test_lengths_and_sealed_blocks(role, n_pending):
    torch_cuda()
    rng = np.random.default_rng(n_pending)
    g, G, hd, cap = 5, 2, 64, 256
    accepted = [-1, 0, 1, g - 1, g, g + 1]  # (below 0 and above gamma: an accept error, nothing is committed)
    B = len(accepted)
    for start in (57, 58, 63):  # (a block is completed by some of them)
        kv = _cache(_shape(hd, G, G, 1), B, cap, 128)
        k, v = (_rows(rng, start + g + 2, G, hd) for _ in range(2))
        for b in range(B):
            kv.write_context(0, b, 0, _bf16(k[:start]), _bf16(v[:start]))
        kv.set_state([start] * B, [[3, 4]] * B, [n_pending] * B)
        new = [np.stack([x[start:]] * B) for x in (k, v)]
        binding.specdec_kv_append(kv, 0, _bf16(new[0]), _bf16(new[1]))
        d, nxt = i32(np.arange(B * g).reshape(B, g) + 100), i32(np.arange(B) + 7)
        binding.specdec_kv_commit(kv, g, role, i32(accepted), d, g, nxt)
        st = kv.read_state()
        log(f"commit role {role} pending {n_pending} from {start}: {st['len'].tolist()}")
        for b, A in enumerate(accepted):
            ok = 0 <= A <= g
            step = 0 if not ok else A + 1 if role == binding.ROLE_TARGET else n_pending + min(A, g - 1)
            n = start + step
            assert st["len"][b] == n
            two = ok and role == binding.ROLE_DRAFT and A == g
            assert st["n_pending"][b] == (n_pending if not ok else 2 if two else 1)
            assert st["pending"][b].tolist() == ([3, 4] if not ok else [100 + b * g + g - 1 if two else 0, 7 + b])
            for got, x in zip(kv.read_context(0, b, 0, n), (k, v)):
                np.testing.assert_array_equal(_np(got), fp8.stored(x[:n], n // 64 * 64))
