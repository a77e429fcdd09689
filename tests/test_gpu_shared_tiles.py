"""Attention over a shared prefix of many sequences, a wave for each 16 of their query rows: one to four tiles of
rows read the same codes, against 64 bits (the bound of test_gpu_shared)."""
import numpy as np
import pytest

from tests.gpu_util import log
from tests.test_gpu_fp8_cache import _cache, _fill, _shape
from tests.test_gpu_shared import _attend, _check, _prefix, _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,H,G,B,n", [(64, 16, 4, 600, 4), (64, 32, 4, 300, 3), (64, 32, 4, 150, 7), (128, 32, 32, 70, 1),
                                        (128, 32, 32, 35, 20), (128, 16, 16, 40, 64), (32, 16, 8, 130, 23)])
def test_tiles_of_many_sequences(hd, H, G, B, n, dtype):
    rng = np.random.default_rng(B + n)
    log(f"tiles hd={hd} H={H} G={G} B={B} n={n} {dtype}")
    prefix, pk, pv = _prefix(rng, hd, G, 150, n_layers=1)
    lens = [int(x) for x in rng.integers(0, 300, B)]
    lens[:4] = [0, 64, 63, 128]
    kv = _cache(_shape(hd, H, G, 1), B, 384, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (B, n, H, hd), dtype)
    log(f"worst error {_check(_attend(prefix, kv, q), q, pk, pv, kvs, lens):.3g}")
