"""Attention over a shared prefix, many bf16 rows of a kv head behind own texts of any length: which kernel
takes a call changes with its sizes, the result does not (against 64 bits, the bound of test_gpu_shared), and
no call takes much longer than the same one of float32 queries, or than one of a few keys less."""
import numpy as np
import pytest

from paper_2608_10362_amd import binding
from tests.gpu_util import log, torch_cuda
from tests.test_gpu_fp8_cache import _bf16, _cache, _fill, _rows, _shape
from tests.test_gpu_shared import _attend, _check, _prefix, _queries

pytestmark = pytest.mark.gpu

# hd, H, G, P, lens, n
CASES = [
    (64, 32, 4, 200, [3000], 3), (64, 32, 4, 65, [4000, 1000], 5), (64, 32, 4, 100, [7000], 9),
    (64, 32, 4, 333, [1500, 20, 3000, 64], 20), (64, 16, 2, 10, [2500] * 3, 65),
    (128, 2, 2, 500, [2500, 8000], 20), (128, 32, 32, 64, [4100], 20), (128, 32, 8, 100, [5000, 1], 9),
    (128, 4, 4, 700, [1000, 6000], 170), (128, 4, 1, 130, [8100], 17),
    (32, 16, 4, 90, [7900, 300], 5), (32, 16, 4, 0, [6000], 100),
    (64, 8, 1, 700, [9000, 12000], 70), (128, 32, 32, 300, [9000] * 2, 70),   # (the second: uncut past 8192 keys)
    (128, 64, 32, 130, [1000] * 8, 35), (64, 64, 16, 64, [900] * 16, 65),     # a wave's rows are its own
    (32, 16, 4, 70, [1500] * 64, 100), (128, 32, 32, 40, [1200] * 24, 68),    # and over longer texts
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"hd{c[0]}h{c[1]}-{c[2]}p{c[3]}b{len(c[4])}l{max(c[4])}n{c[5]}")
def test_many_rows_over_longer_texts(case):
    hd, H, G, P, lens, n = case
    rng = np.random.default_rng(P + n + hd)
    log(f"shared, longer own texts {case}")
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), len(lens), (max(lens) + n + 63) // 64 * 64, (n + 63 + 63) // 64 * 64 + 64)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (len(lens), n, H, hd), "bf16")
    log(f"worst error {_check(_attend(prefix, kv, q), q, pk, pv, kvs, lens):.3g}")


@pytest.mark.parametrize("P", [40, 1000])
@pytest.mark.parametrize("hd,H,G,B,n,L", [(128, 8, 8, 2, 70, 700), (64, 32, 4, 1, 9, 3000), (64, 64, 16, 16, 65, 700),
                                          (128, 64, 32, 8, 35, 700), (32, 16, 4, 64, 100, 1500)])
def test_maxima_that_rise_from_chunk_to_chunk(hd, H, G, B, n, L, P):
    """Keys whose scores grow along the text, from a prefix that lies far below: every chunk raises the maxima."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd + L + P)
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), B, (L + n + 63) // 64 * 64, 256)
    q = _queries(rng, (B, n, H, hd), "bf16", 0.5)
    q[..., 0] = 4.0
    from oracle import fp8
    kvs = []
    new = [np.zeros((B, n, G, hd), np.float32) for _ in range(2)]
    for b in range(B):
        k, v = _rows(rng, L + n, G, hd, False), _rows(rng, L + n, G, hd, False)
        k[:, :, 0] = (np.arange(L + n) / (L + n) * 40.0)[:, None]  # (scores up to 160 / sqrt(hd) above the first)
        k, v = (x.astype(np.float32) for x in (k, v))
        kb, vb = (_bf16(x) for x in (k, v))
        kv.write_context(0, b, 0, kb[:L].contiguous(), vb[:L].contiguous())
        k, v = (x.float().cpu().numpy() for x in (kb, vb))
        new[0][b], new[1][b] = k[L:], v[L:]
        kvs.append((fp8.stored(k, L // 64 * 64), fp8.stored(v, L // 64 * 64)))
    kv.set_state([L] * B, [[0, 1]] * B, [1] * B)
    binding.specdec_kv_append(kv, 0, _bf16(new[0]), _bf16(new[1]))
    log(f"rising maxima hd={hd} B={B} n={n} L={L} P={P}")
    _check(_attend(prefix, kv, q), q, pk, pv, kvs, [L] * B)


@pytest.mark.parametrize("hd,H,G,n", [(64, 32, 4, 5), (128, 8, 8, 70), (64, 32, 4, 9)])
def test_replays_at_other_lengths(hd, H, G, n):
    """Captured for texts of 6000 keys, replayed at shorter ones; two graphs of one workspace in turn."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd + n)
    prefix, pk, pv = _prefix(rng, hd, G, 300, n_layers=1)
    cap = 6144
    kv = [_cache(_shape(hd, H, G, 1), 2, cap, 256) for _ in range(2)]
    q = [_queries(rng, (2, n, H, hd), "bf16") for _ in kv]
    out = [torch.empty_like(x) for x in q]
    ws = binding.shared_attention_workspace(prefix, kv[0], H, n, torch.bfloat16)
    ws.fill_(255)
    graphs = []
    for c, x, o in zip(kv, q, out):
        c.kv.len_upper = 6000
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.specdec_attention_shared(prefix, c, 0, x, o, ws, 1)
        graphs.append(g)
    for lens in ([6000, 64], [10, 4100], [0, 2500], [5900, 5999]):
        held = [_fill(c, rng, lens, n, G, hd) for c in kv]
        log(f"replays hd={hd} n={n} lengths {lens}")
        for _ in range(2):
            for o in out:
                o.fill_(float("nan"))
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            for i, c in enumerate(kv):
                _check(out[i], q[i], pk, pv, held[i], lens)
                assert c.read_state()["status"] == 0


def _best_us(hd, H, G, B, n, L, dtype):
    """The fastest of six rounds of calls, microseconds (sums and codes of any values: the caches are filled with one row)."""
    torch = torch_cuda()
    kv = _cache(_shape(hd, H, G, 1), B, (L + n + 63) // 64 * 64, (n + 63 + 63) // 64 * 64 + 64)
    prefix = _cache(_shape(hd, H, G, 1), 1, 256, 128)
    rows = torch.randn((L, G, hd), device="cuda").bfloat16()
    for b in range(B):
        kv.write_context(0, b, 0, rows, rows)
    prefix.write_context(0, 0, 0, rows[:200].contiguous(), rows[:200].contiguous())
    prefix.set_state([200], [[0, 1]], [1])
    kv.set_state([L] * B, [[0, 1]] * B, [1] * B)
    x = torch.randn((B, n, G, hd), device="cuda").bfloat16()
    binding.specdec_kv_append(kv, 0, x, x)
    q = torch.randn((B, n, H, hd), device="cuda").to(dtype)
    out, ws = torch.empty_like(q), binding.shared_attention_workspace(prefix, kv, H, n, dtype)
    best = float("inf")
    for _ in range(6):
        at = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        at[0].record()
        for _ in range(10):
            binding.specdec_attention_shared(prefix, kv, 0, q, out, ws)
        at[1].record()
        torch.cuda.synchronize()
        best = min(best, at[0].elapsed_time(at[1]) * 100)
    return best


@pytest.mark.parametrize("hd,H,G,B,n,L", [(64, 32, 4, 1, 5, 8000), (64, 32, 4, 16, 3, 8000), (64, 32, 4, 16, 9, 4000),
                                          (128, 32, 32, 1, 20, 8000), (128, 32, 32, 2, 20, 8000), (128, 32, 32, 2, 40, 8000),
                                          (128, 32, 32, 1, 170, 8000), (128, 32, 32, 2, 70, 2500)])
def test_bf16_takes_no_longer_than_float32(hd, H, G, B, n, L):
    torch = torch_cuda()
    half, full = (_best_us(hd, H, G, B, n, L, t) for t in (torch.bfloat16, torch.float32))
    log(f"hd={hd} G={G} B={B} n={n} L={L}: bf16 {half:.0f} us, float32 {full:.0f} us")
    assert half <= 1.6 * full + 8  # (above the spread of such times; a wrong choice cost 1.9 to 5.6 times)


@pytest.mark.parametrize("hd,H,G,B,n", [(64, 32, 4, 16, 3), (128, 32, 32, 32, 40), (128, 32, 8, 64, 17), (64, 32, 4, 2, 20)])
def test_a_few_keys_more_take_little_longer(hd, H, G, B, n):
    torch = torch_cuda()
    less, more = (_best_us(hd, H, G, B, n, L, torch.bfloat16) for L in (8064, 8256))
    log(f"hd={hd} G={G} B={B} n={n}: 8064 keys {less:.0f} us, 8256 {more:.0f} us")
    assert max(less, more) <= 1.6 * min(less, more) + 8
