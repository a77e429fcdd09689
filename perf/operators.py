"""The serving operators this library's speed is judged by, and what each returns.

Three operators a serving loop adds to the draft-and-verify iteration:

  sample    logits -> the distribution left by a request's rules (temperature,
            min-p, top-k, top-p) and a token drawn from it with a given word;
            the accept rule takes such distributions, a plain loop the token
  attend    grouped-query attention of the newest positions over a cache whose
            blocks of 64 positions are held in 8 bits (e4m3 codes and one
            power-of-two scale per block, kv head, and K or V; the newest,
            incomplete block and the new rows are bfloat16)
  exchange  a sequence's keys and values written into such a cache and read
            back (a parked or moved request: quantize, then dequantize)

Shapes are the 7B-like and the 1.1B-like decoder of synth.py; keys and values
are N(0, (0.02 sqrt d)^2) as its contexts are, queries N(0, 1), logits
N(0, 2.5^2) with a few likely tokens raised.  With `own` the operators are the
library's; without it they are elementary torch operations.

Cases are plain dicts:
  op       sample | attend | exchange
  batch, rows, vocab, rules, probs      sample (rules: top_k | top_p | mixed | plain)
  shape, batch, ctx_lo, ctx_hi, new     attend: committed lengths, new rows a sequence
  shape, positions                      exchange
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 64      # positions of one scale
E4M3_MAX = 448.0
MIN_EXP = -100  # smallest scale exponent
SHAPES = {  # heads, kv heads, head dim, model width
    "7b": (32, 32, 128, 4096),
    "1b": (32, 4, 64, 2048),
}


# ---------------------------------------------------------------- the cases
def _sample(name, batch, rows, vocab, rules, probs):
    return {"name": name, "op": "sample", "batch": batch, "rows": rows, "vocab": vocab, "rules": rules, "probs": probs}


def _attend(name, shape, batch, ctx_lo, ctx_hi, new):
    return {"name": name, "op": "attend", "shape": shape, "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "new": new}


def _exchange(name, shape, positions):
    return {"name": name, "op": "exchange", "shape": shape, "positions": positions}


def listed():
    return [
        # the next token of one stream: the smallest sampling call
        _sample("sample_b1_32k", 1, 1, 32000, "top_k", False),
        # the target rows of a verify pass of four streams, each with rules of its own, for the accept rule
        _sample("sample_b4_g4_32k", 4, 5, 32000, "mixed", True),
        # the next tokens of a full batch over a large vocabulary, nucleus sampling
        _sample("sample_b16_128k", 16, 1, 128256, "top_p", False),
        # the target rows of a full batch's verify pass over a large vocabulary: the largest sampling call
        _sample("sample_b16_g6_128k", 16, 7, 128256, "mixed", True),
        # one stream decoding one token at an ordinary context, one query head a kv head
        _attend("attend_7b_b1", "7b", 1, 2047, 2047, 1),
        # a verify pass of four ragged streams with grouped queries
        _attend("attend_1b_b4_g4", "1b", 4, 301, 1023, 5),
        # one long document, grouped queries: work split over the keys
        _attend("attend_1b_long", "1b", 1, 131071, 131071, 1),
        # a batch of long ragged streams decoding: the key and value stream
        _attend("attend_7b_b16", "7b", 16, 1024, 8190, 1),
        # a prompt's last chunk over the chunks before it: the products
        _attend("attend_7b_chunk", "7b", 1, 1536, 1536, 512),
        # a short prompt parked and brought back
        _exchange("exchange_1b_130", "1b", 130),
        # an ordinary conversation
        _exchange("exchange_7b_2k", "7b", 2048),
        # a long one, ending inside a block
        _exchange("exchange_7b_32k", "7b", 32745),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "attend", "attend", "attend", "exchange"])
    if op == "sample":
        batch, rows = _log(rng, 1, 16), rng.choice([1, 1, rng.randint(2, 7)])
        c = _sample("", batch, rows, _log(rng, 2000, 128256), rng.choice(["top_k", "top_p", "mixed", "plain"]),
                    rng.random() < 0.5)
    elif op == "attend":
        shape = rng.choice(["7b", "1b"])
        batch, new = _log(rng, 1, 16), rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 400)])
        if new > 9:
            batch = min(batch, 2) if new < 100 else 1
        hi = _log(rng, 1, 60000 // batch if shape == "7b" else 120000 // batch) if new <= 9 else _log(rng, 1, 2000)
        c = _attend("", shape, batch, rng.randint(max(1, hi // 8), hi), hi, new)
    else:
        c = _exchange("", rng.choice(["7b", "1b"]), _log(rng, 1, 30000))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, idx):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + idx) & 0x7FFFFFFFFFFF)
    return g


def _normal(seed, idx, shp, sigma, dtype=torch.float32):
    return torch.empty(shp, dtype=torch.float32, device=DEV).normal_(0.0, sigma, generator=_gen(seed, idx)).to(dtype)


def _lengths(case):
    """Committed lengths, spread evenly over the batch in a scattered order."""
    B, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    if B == 1:
        return [hi]
    step = 7 if B % 7 else 1
    return [lo + (hi - lo) * ((step * b + 3) % B) // (B - 1) for b in range(B)]


def _rules(case, seed):
    """Per-sequence rules (temperature, top_k, top_p, min_p); None: not given."""
    B, kind = case["batch"], case["rules"]
    r = np.random.RandomState((int(seed) * 7919 + 17) & 0x7FFFFFFF)
    t = torch.tensor(r.choice([0.6, 0.7, 0.8, 1.0], B), dtype=torch.float32, device=DEV)
    k = torch.tensor(r.choice([1, 20, 40, 50, 64, 1000], B), dtype=torch.int32, device=DEV)
    p = torch.tensor(r.choice([0.7, 0.8, 0.9, 0.95, 0.99], B), dtype=torch.float32, device=DEV)
    if kind == "top_k":
        return t, k, None, None
    if kind == "top_p":
        return t, None, p, None
    if kind == "plain":
        return t, None, None, None
    on = r.rand(3, B) < 0.6  # a request sets some of the rules
    k = torch.where(torch.tensor(on[0], device=DEV), k, torch.zeros_like(k))
    p = torch.where(torch.tensor(on[1], device=DEV), p, torch.ones_like(p))
    mp = torch.tensor(np.where(on[2], r.choice([0.02, 0.05, 0.1], B), 0.0), dtype=torch.float32, device=DEV)
    return t, k, p, mp


def _pow2_scale(amax):
    """2^e, e the smallest integer >= MIN_EXP with amax <= 448 * 2^e."""
    _, e = torch.frexp(amax.double() / E4M3_MAX)  # amax / 448 = f * 2^e, f in [0.5, 1)
    e = torch.where(amax.double() <= E4M3_MAX * torch.exp2(e.double() - 1), e - 1, e)
    e = torch.where(amax == 0, torch.full_like(e, MIN_EXP), e).clamp(min=MIN_EXP)
    return torch.exp2(e.double()).float()


def _quantize(x):
    """[..., positions % 64 == 0, G, hd] bfloat16 -> e4m3 codes and scales [..., blocks, G]."""
    shp = x.shape
    xb = x.float().reshape(*shp[:-3], shp[-3] // BLOCK, BLOCK, *shp[-2:])
    s = _pow2_scale(xb.abs().amax(dim=(-1, -3)))
    return (xb / s[..., None, :, None]).to(torch.float8_e4m3fn).reshape(shp), s


def _dequantize(c, s):
    shp = c.shape
    cb = c.float().reshape(*shp[:-3], shp[-3] // BLOCK, BLOCK, *shp[-2:])
    return (cb * s[..., None, :, None]).reshape(shp)


def _round_up(n, m):
    return -(-n // m) * m


def prepare(case, seed):
    st = {"case": case, "seed": int(seed)}
    if case["op"] == "sample":
        B, R, V = case["batch"], case["rows"], case["vocab"]
        lg = _normal(seed, 1, (B, R, V), 2.5)
        top = torch.randint(0, V, (B, R, 12), device=DEV, generator=_gen(seed, 2))
        lg.scatter_(-1, top, 9.0 + 1.5 * _normal(seed, 3, (B, R, 12), 1.0))
        if case["rules"] == "mixed":  # a grammar forbids part of the first sequence's vocabulary
            lg[0].masked_fill_(torch.rand((R, V), device=DEV, generator=_gen(seed, 4)) < 0.7, -math.inf)
        st["logits"], st["rules"] = lg, _rules(case, seed)
        st["words"] = torch.randint(-2 ** 31, 2 ** 31, (B, R), dtype=torch.int64, device=DEV,
                                    generator=_gen(seed, 5)).to(torch.int32)
        if own:
            from paper_2608_10362_amd import binding
            t, k, p, mp = st["rules"]
            st["own_rules"] = binding.SamplingRules(temperature=t, top_k=k, top_p=p, min_p=mp)
            st["out"] = torch.empty((B, R), dtype=torch.int32, device=DEV)
            st["probs"] = torch.empty((B, R, V), dtype=torch.float32, device=DEV) if case["probs"] else None
            st["ws"] = binding.sample_workspace(B, R, V, DEV)
        return st
    H, G, hd, d = SHAPES[case["shape"]]
    sigma = 0.02 * d ** 0.5
    if case["op"] == "exchange":
        n = case["positions"]
        st["k"] = _normal(seed, 11, (n, G, hd), sigma, torch.bfloat16)
        st["v"] = _normal(seed, 12, (n, G, hd), sigma, torch.bfloat16)
        if own:
            st["kv"] = _own_cache(case["shape"], 1, _round_up(n, BLOCK), 128)
            st["kv"].set_state([n], [[0, 1]], [1])
        return st
    B, n, lens = case["batch"], case["new"], _lengths(case)
    cap = _round_up(max(lens) + n, BLOCK)
    k = _normal(seed, 21, (B, cap, G, hd), sigma, torch.bfloat16)
    v = _normal(seed, 22, (B, cap, G, hd), sigma, torch.bfloat16)
    st["q"] = _normal(seed, 23, (B, n, H, hd), 1.0)
    st["len"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    # the cache: codes and scales of every block (those past a sequence's last whole one are not read), and the rows
    # from its last whole block on in bfloat16
    (st["kc"], st["ks"]), (st["vc"], st["vs"]) = _quantize(k), _quantize(v)
    tail = BLOCK + n
    at = (st["len"] // BLOCK * BLOCK)[:, None].long() + torch.arange(tail, device=DEV)[None]
    at = at.clamp(max=cap - 1)[:, :, None, None].expand(-1, -1, G, hd)
    st["kt"], st["vt"] = torch.gather(k, 1, at), torch.gather(v, 1, at)
    if own:
        from paper_2608_10362_amd import binding
        st["kv"] = kv = _own_cache(case["shape"], B, cap, _round_up(BLOCK + n, BLOCK))
        for b in range(B):
            kv.write_context(0, b, 0, k[b, :lens[b]].contiguous(), v[b, :lens[b]].contiguous())
        kv.set_state(lens, [[0, 1]] * B, [1] * B)
        rows = (st["len"][:, None].long() + torch.arange(n, device=DEV)[None])[:, :, None, None].expand(-1, -1, G, hd)
        binding.specdec_kv_append(kv, 0, torch.gather(k, 1, rows).contiguous(), torch.gather(v, 1, rows).contiguous())
        st["ws"] = binding.attention_workspace(kv, H, n)
        st["out"] = torch.empty((B, n, H, hd), dtype=torch.float32, device=DEV)
    return st


def _own_cache(shape, batch, capacity, window):
    from paper_2608_10362_amd import binding, synth
    s = {"7b": synth.LLAMA_7B, "1b": synth.LLAMA_1B}[shape]
    return binding.Fp8KVCache(s, batch, capacity, window, n_layers=1, device=DEV)


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    if case["op"] == "sample":
        probs, tokens = _plain_sample(st["logits"], st["rules"], st["words"])
        return {"probs": probs, "tokens": tokens} if case["probs"] else {"tokens": tokens}
    if case["op"] == "attend":
        return {"out": _plain_attend(st)}
    return {"k": _plain_exchange(st["k"]), "v": _plain_exchange(st["v"])}


def _run_own(case, st):
    from paper_2608_10362_amd import binding
    if case["op"] == "sample":
        binding.specdec_sample_logits(st["logits"], st["own_rules"], rand=st["words"], probs=st["probs"], out=st["out"],
                                      workspace=st["ws"])
        return {"probs": st["probs"], "tokens": st["out"]} if case["probs"] else {"tokens": st["out"]}
    if case["op"] == "attend":
        binding.specdec_attention(st["kv"], 0, st["q"], st["out"], st["ws"])
        return {"out": st["out"]}
    st["kv"].write_context(0, 0, 0, st["k"], st["v"])
    k, v = st["kv"].read_context(0, 0, 0, case["positions"])
    return {"k": k, "v": v}


def _plain_sample(logits, rules, words):
    B, R, V = logits.shape
    t, k, p, mp = rules
    col = lambda x: x.reshape(B, 1, 1)  # noqa: E731
    m = logits.amax(-1, keepdim=True).double()
    e = torch.exp((logits.double() - m) / col(t).double())
    if mp is not None:
        e = torch.where(e >= col(mp).double(), e, torch.zeros_like(e))
    # descending, ties by index (a stable sort keeps their order); dropped entries have weight 0 and go last
    key = torch.where(e > 0, logits, torch.full_like(logits, -math.inf))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    es = torch.gather(e, -1, order)
    n = (e > 0).sum(-1, keepdim=True)
    if k is not None:
        n = torch.where(col(k) > 0, torch.minimum(n, col(k).long()), n)
    c = torch.cumsum(torch.floor(es * 2.0 ** 43).long(), -1)
    ck = torch.gather(c, -1, n - 1)
    if p is not None:
        need = torch.ceil(col(p).double() * ck.double()).long().clamp(min=1)
        n = torch.where(col(p) < 1, torch.minimum(n, (c < need).sum(-1, keepdim=True) + 1), n)
        ck = torch.gather(c, -1, n - 1)
    keep = torch.arange(V, device=logits.device) < n
    ps = torch.where(keep, es * 2.0 ** 43 / ck.double(), torch.zeros_like(es)).float()
    probs = torch.empty_like(logits).scatter_(-1, order, ps)
    # fixed-point draw: t = floor(x S / 2^32) with x in 16-bit halves
    cum = torch.cumsum(torch.floor(probs.double() * 2.0 ** 40).long(), -1)
    S, x = cum[..., -1], words.long() & 0xFFFFFFFF
    at = ((x >> 16) * S + (((x & 0xFFFF) * S) >> 16)) >> 16
    return probs, (cum <= at[..., None]).sum(-1).to(torch.int32)


def _plain_attend(st):
    q, n_len = st["q"], st["len"].long()
    B, n, H, hd = q.shape
    G, cap, tail = st["kc"].shape[2], st["kc"].shape[1], st["kt"].shape[1]
    sealed = n_len // BLOCK * BLOCK
    k = torch.cat([_dequantize(st["kc"], st["ks"]), st["kt"].float()], 1)
    v = torch.cat([_dequantize(st["vc"], st["vs"]), st["vt"].float()], 1)
    # positions of the keys: a code counts below the last whole block's end, a tail row at its place
    i, j = torch.arange(cap, device=q.device)[None], torch.arange(tail, device=q.device)[None]
    far = torch.full((), 1 << 40, device=q.device)
    pos = torch.cat([torch.where(i < sealed[:, None], i, far), sealed[:, None] + j], 1)
    seen = pos[:, None] <= (n_len[:, None] + torch.arange(n, device=q.device))[:, :, None]
    qg = q.reshape(B, n, G, H // G, hd).permute(0, 2, 1, 3, 4).reshape(B, G, n * (H // G), hd)
    s = torch.matmul(qg, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(hd))
    s = s.reshape(B, G, n, H // G, -1).masked_fill(~seen[:, None, :, None], -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(e.reshape(B, G, n * (H // G), -1), v.transpose(1, 2).contiguous())
    o = o.reshape(B, G, n, H // G, hd) / e.sum(-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, H, hd).contiguous()


def _plain_exchange(x):
    whole = x.shape[0] // BLOCK * BLOCK
    return torch.cat([_dequantize(*_quantize(x[:whole])).to(torch.bfloat16), x[whole:]])


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        rows = case["batch"] * case["rows"]
        n = float(rows) * case["vocab"]
        return {"bytes": n * (8.0 if case["probs"] else 4.0) + 8.0 * rows, "flops": 4.0 * n}
    H, G, hd, _ = SHAPES[case["shape"]]
    if case["op"] == "exchange":
        n = case["positions"]
        whole = n // BLOCK * BLOCK
        return {"bytes": 2.0 * G * hd * (whole * 6 + (n - whole) * 8), "flops": 2.0 * G * hd * n * 4}
    n, nbytes, pairs = case["new"], 0.0, 0.0
    for L in _lengths(case):
        sealed = L // BLOCK * BLOCK
        nbytes += 2.0 * G * hd * (sealed + 2.0 * (L + n - sealed)) + 8.0 * n * H * hd
        pairs += n * L + n * (n + 1) / 2
    return {"bytes": nbytes, "flops": 4.0 * H * hd * pairs}


# ---------------------------------------------------------------- 64-bit results
def _kept_row(l, t, k, p, mp):
    """The kept tokens of one row of logits (numpy float64), most likely first."""
    z = (l - l.max()) / t
    idx = np.flatnonzero(np.isfinite(l) & (np.exp(z) >= mp))
    idx = idx[np.lexsort((idx, -l[idx]))]
    if k > 0:
        idx = idx[:k]
    if p < 1:
        mass = np.floor(np.exp(z[idx]) * 2.0 ** 43).astype(np.int64)
        need = max(1, math.ceil(p * float(mass.sum())))
        idx = idx[:int(np.searchsorted(np.cumsum(mass), need)) + 1]
    return idx, z


def _e4m3(x):
    """Nearest e4m3 value of |x| <= 448 (float64), ties to even: 3 mantissa bits, smallest exponent -6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_blocks(x):
    """[n, G, hd] bfloat16 -> what the cache's whole blocks stand for, and the rows after them, in 64 bits."""
    x = x.double()
    whole = x.shape[0] // BLOCK * BLOCK
    xb = x[:whole].reshape(whole // BLOCK, BLOCK, *x.shape[1:])
    amax = xb.abs().amax(dim=(1, 3), keepdim=True).clamp(min=2.0 ** -140)
    s = torch.exp2(torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(min=MIN_EXP))
    return torch.cat([(_e4m3(xb / s) * s).reshape(whole, *x.shape[1:]), x[whole:]])


def exact(case, seed):
    st = prepare(dict(case), seed)
    if case["op"] == "sample":
        if not case["probs"]:
            return None  # whole numbers, decided by integer sums
        B, R, V = st["logits"].shape
        t, k, p, mp = (None if r is None else r.double().cpu().numpy() for r in st["rules"])
        l, out = st["logits"].double().cpu().numpy(), np.zeros((B, R, V))
        for b in range(B):
            for i in range(R):
                idx, z = _kept_row(l[b, i], t[b], int(k[b]) if k is not None else 0, p[b] if p is not None else 1.0,
                                   mp[b] if mp is not None else 0.0)
                e = np.exp(z[idx])
                out[b, i, idx] = e / e.sum()
        return {"probs": torch.from_numpy(out), "tokens": None}
    H, G, hd, d = SHAPES[case["shape"]]
    sigma = 0.02 * d ** 0.5
    if case["op"] == "exchange":
        return {"k": _exact_blocks(st["k"]), "v": _exact_blocks(st["v"])}
    B, n, lens = case["batch"], case["new"], _lengths(case)
    cap = _round_up(max(lens) + n, BLOCK)
    k = _normal(seed, 21, (B, cap, G, hd), sigma, torch.bfloat16)
    v = _normal(seed, 22, (B, cap, G, hd), sigma, torch.bfloat16)
    out = torch.empty((B, n, H, hd), dtype=torch.float64, device=DEV)
    r = H // G
    for b in range(B):
        m = lens[b] + n
        whole = lens[b] // BLOCK * BLOCK
        kb = torch.cat([_exact_blocks(k[b, :whole]), k[b, whole:m].double()])
        vb = torch.cat([_exact_blocks(v[b, :whole]), v[b, whole:m].double()])
        late = torch.arange(m, device=DEV)[None] > lens[b] + torch.arange(n, device=DEV)[:, None]
        for h in range(H):
            s = (st["q"][b, :, h].double() @ kb[:, h // r].t().contiguous()) / math.sqrt(hd)
            out[b, :, h] = torch.softmax(s.masked_fill(late, -math.inf), -1) @ vb[:, h // r].contiguous()
    return {"out": out}
