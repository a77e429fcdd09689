"""More serving operators this library's speed is judged by, and what each returns.

The attention block of a caller's own model over 8-bit caches, from the
projections to the attention's output, for a batch whose requests start with
the same text:

  rotate  queries and keys of every head: RMS norm with a gain, then the
          rotation of their position; in and out as tensors (a model with a
          cache of its own)
  append  the same, the keys and the values written into an 8-bit cache's
          newest rows in that pass, the queries handed to the attention; the
          rows are read back
  shared  attention of the newest rows of every sequence over a prefix that is
          held once, for all of them, and over the sequence's own cache

Shapes are the 7B-like and the 1.1B-like decoder of synth.py.  Projections are
N(0, (0.02 sqrt d)^2) as rows of weights N(0, 0.02^2) leave of normalised
inputs, keys and values of the caches the same, queries N(0, 1), gains near 1.
With `own` the operators are the library's; without it they are elementary
torch operations.

Cases are plain dicts:
  op       rotate | append | shared
  shape, batch, rows, start             rotate, append: rows a sequence, the first one's position
                                        (append: committed lengths, spread below `start`)
  rotary, interleaved, norm             dims rotated, pairs side by side or half of them apart, norm or not
  dtype, out                            types of the projections, and of the queries (rotate: and keys)
  shape, batch, prefix, lo, hi, new     shared: lengths of the prefix and of the sequences' own text, new rows
  dtype                                 type of the queries and the result
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 64      # positions of one scale
E4M3_MAX = 448.0
MIN_EXP = -100  # smallest scale exponent
BASE = 10000.0  # of the rotation's angles
EPS = 1e-5
SHAPES = {  # heads, kv heads, head dim, model width
    "7b": (32, 32, 128, 4096),
    "1b": (32, 4, 64, 2048),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- the cases
def _rotate(name, shape, batch, rows, start, rotary, interleaved, norm, dtype, out):
    return {"name": name, "op": "rotate", "shape": shape, "batch": batch, "rows": rows, "start": start,
            "rotary": rotary, "interleaved": interleaved, "norm": norm, "dtype": dtype, "out": out}


def _append(name, shape, batch, rows, start, rotary, interleaved, norm, dtype, out):
    return {**_rotate(name, shape, batch, rows, start, rotary, interleaved, norm, dtype, out), "op": "append"}


def _shared(name, shape, batch, prefix, lo, hi, new, dtype):
    return {"name": name, "op": "shared", "shape": shape, "batch": batch, "prefix": prefix, "lo": lo, "hi": hi,
            "new": new, "dtype": dtype}


def listed():
    return [
        # the next token of one stream: the smallest call
        _rotate("rotate_7b_b1", "7b", 1, 1, 4095, 128, False, True, "bf16", "bf16"),
        # the newest tokens of a full batch, far along, half of each head rotated in pairs side by side
        _rotate("rotate_1b_b96", "1b", 96, 1, 900001, 32, True, True, "bf16", "f32"),
        # a long prompt at once
        _rotate("rotate_7b_8k", "7b", 1, 8189, 0, 128, False, True, "bf16", "bf16"),
        # a verify pass of four ragged streams: float32 projections, no norm
        _append("append_1b_b4_g4", "1b", 4, 5, 1023, 64, False, False, "f32", "f32"),
        # a prompt's chunk behind the chunks before it
        _append("append_7b_2k", "7b", 1, 2048, 4096, 128, False, True, "bf16", "bf16"),
        # two short questions to one system prompt: the smallest attention
        _shared("shared_1b_b2", "1b", 2, 200, 1, 40, 1, "f32"),
        # a batch of chats with one system prompt and examples, decoding
        _shared("shared_7b_b16", "7b", 16, 8192, 64, 700, 1, "bf16"),
        # a verify pass of such a batch, in the types of the library's own passes
        _shared("shared_7b_b16_g4", "7b", 16, 4001, 0, 512, 5, "f32"),
        # many questions to one book: grouped queries
        _shared("shared_1b_b64_64k", "1b", 64, 65553, 30, 300, 1, "bf16"),
        # a large batch of samples from one long context: the products
        _shared("shared_7b_b128_16k", "7b", 128, 16384, 0, 256, 1, "bf16"),
        # several prompts that begin alike, the chunk after what they share
        _shared("shared_7b_b6_chunk", "7b", 6, 3500, 0, 0, 170, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "shared", "shared", "shared"])
    shape = rng.choice(["7b", "1b"])
    hd = SHAPES[shape][2]
    if op == "shared":
        batch, new = _log(rng, 1, 128), rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 170)])
        new = min(new, max(1, 1020 // batch))
        prefix = _log(rng, 1, 65536 if shape == "1b" else 20000)
        if batch * new > 64 and shape == "7b":
            prefix = max(1, min(prefix, 2000000 // (batch * new)))
        if batch * new > 64 and shape == "1b":
            prefix = max(1, min(prefix, 4000000 // (batch * new)))
        hi = _log(rng, 1, max(2, 60000 // batch if new < 10 else 600))
        c = _shared("", shape, batch, prefix, rng.randint(0, hi), hi, new, rng.choice(["bf16", "bf16", "f32"]))
    else:
        batch = _log(rng, 1, 128) if op == "rotate" else rng.randint(1, 4)
        rows = _log(rng, 1, 8189 // batch) if op == "rotate" else rng.choice([1, rng.randint(2, 9), _log(rng, 10, 2048)])
        make = _rotate if op == "rotate" else _append
        start = _log(rng, 1, 1000000) if op == "rotate" else _log(rng, 1, 8000)
        c = make("", shape, batch, rows, start, rng.choice([hd, hd, hd // 2, 16]), rng.random() < 0.4, rng.random() < 0.7,
                 rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"]))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, idx):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + idx) & 0x7FFFFFFFFFFF)
    return g


def _normal(seed, idx, shp, sigma, dtype=torch.float32):
    return torch.empty(shp, dtype=torch.float32, device=DEV).normal_(0.0, sigma, generator=_gen(seed, idx)).to(dtype)


def _spread(n, lo, hi):
    """n lengths, spread evenly over lo .. hi in a scattered order."""
    if n == 1:
        return [hi]
    step = 7 if n % 7 else 1
    return [lo + (hi - lo) * ((step * b + 3) % n) // (n - 1) for b in range(n)]


def _starts(case):
    """The position of each sequence's first row."""
    return _spread(case["batch"], case["start"] // 3, case["start"])


def _lengths(case):
    return _spread(case["batch"], case["lo"], case["hi"])


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


def _projections(case, seed):
    """q, k, v: three views of the rows a fused projection leaves."""
    H, G, hd, d = SHAPES[case["shape"]]
    B, n = case["batch"], case["rows"]
    x = _normal(seed, 1, (B, n, (H + 2 * G) * hd), 0.02 * d ** 0.5, TYPES[case["dtype"]])
    q, k, v = x.split([H * hd, G * hd, G * hd], -1)
    return q.unflatten(-1, (H, hd)), k.unflatten(-1, (G, hd)), v.unflatten(-1, (G, hd))


def _gains(case, seed):
    hd = SHAPES[case["shape"]][2]
    if not case["norm"]:
        return None, None
    return tuple((1.0 + _normal(seed, i, (hd,), 0.1)).to(TYPES[case["dtype"]]) for i in (2, 3))


def _prefix_rows(case, seed):
    H, G, hd, d = SHAPES[case["shape"]]
    cap = _round_up(case["prefix"], BLOCK)
    return tuple(_normal(seed, i, (cap, G, hd), 0.02 * d ** 0.5, torch.bfloat16) for i in (11, 12))


def _own_rows(case, seed):
    """Keys and values of the sequences' own text, the new rows behind each length."""
    H, G, hd, d = SHAPES[case["shape"]]
    cap = _round_up(max(_lengths(case)) + case["new"], BLOCK)
    return tuple(_normal(seed, i, (case["batch"], cap, G, hd), 0.02 * d ** 0.5, torch.bfloat16) for i in (21, 22))


def prepare(case, seed):
    st = {"case": case}
    H, G, hd, d = SHAPES[case["shape"]]
    B = case["batch"]
    if case["op"] != "shared":
        n = case["rows"]
        st["q"], st["k"], st["v"] = _projections(case, seed)
        st["gains"] = _gains(case, seed)
        starts = _starts(case)
        st["pos"] = (torch.tensor(starts, dtype=torch.int32, device=DEV)[:, None] +
                     torch.arange(n, dtype=torch.int32, device=DEV)[None])
        st["q_out"] = torch.empty((B, n, H, hd), dtype=TYPES[case["out"]], device=DEV)
        if own:
            from paper_2608_10362_amd import binding
            st["rope"] = binding.Rope(hd, rotary_dim=case["rotary"], base=BASE, interleaved=case["interleaved"],
                                      q_gain=st["gains"][0], k_gain=st["gains"][1], eps=EPS)
            if case["op"] == "append":
                st["starts"] = starts
                st["kv"] = _own_cache(case["shape"], B, _round_up(max(starts) + n, BLOCK), _round_up(n + 63, BLOCK))
                st["kv"].set_state(starts, [[0, 1]] * B, [1] * B)
            else:
                st["k_out"] = torch.empty((B, n, G, hd), dtype=TYPES[case["out"]], device=DEV)
        return st
    n, P, lens = case["new"], case["prefix"], _lengths(case)
    (pk, pv), (k, v) = _prefix_rows(case, seed), _own_rows(case, seed)
    cap = k.shape[1]
    st["q"] = _normal(seed, 31, (B, n, H, hd), 1.0, TYPES[case["dtype"]])
    st["len"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    rows = (st["len"][:, None].long() + torch.arange(n, device=DEV)[None])[:, :, None, None].expand(-1, -1, G, hd)
    if own:
        from paper_2608_10362_amd import binding
        st["prefix"] = _own_cache(case["shape"], 1, _round_up(P, BLOCK), 128)
        st["prefix"].write_context(0, 0, 0, pk[:P], pv[:P])
        st["prefix"].set_state([P], [[0, 1]], [1])
        st["kv"] = kv = _own_cache(case["shape"], B, cap, max(128, _round_up(n + 63, BLOCK)))
        for b in range(B):
            if lens[b]:
                kv.write_context(0, b, 0, k[b, :lens[b]].contiguous(), v[b, :lens[b]].contiguous())
        kv.set_state(lens, [[0, 1]] * B, [1] * B)
        binding.specdec_kv_append(kv, 0, torch.gather(k, 1, rows).contiguous(), torch.gather(v, 1, rows).contiguous())
        st["ws"] = binding.shared_attention_workspace(st["prefix"], kv, H, n, dtype=st["q"].dtype)
        st["out"] = torch.empty_like(st["q"])
        return st
    # the caches: codes and scales of whole blocks, the rows behind the last of them in bfloat16
    (st["pkc"], st["pks"]), (st["pvc"], st["pvs"]) = _quantize(pk), _quantize(pv)
    whole = P // BLOCK * BLOCK
    st["pkt"], st["pvt"] = pk[whole:P].clone(), pv[whole:P].clone()
    (st["kc"], st["ks"]), (st["vc"], st["vs"]) = _quantize(k), _quantize(v)
    tail = BLOCK + n
    at = (st["len"] // BLOCK * BLOCK)[:, None].long() + torch.arange(tail, device=DEV)[None]
    at = at.clamp(max=cap - 1)[:, :, None, None].expand(-1, -1, G, hd)
    st["kt"], st["vt"] = torch.gather(k, 1, at), torch.gather(v, 1, at)
    return st


def _own_cache(shape, batch, capacity, window):
    from paper_2608_10362_amd import binding, synth
    s = {"7b": synth.LLAMA_7B, "1b": synth.LLAMA_1B}[shape]
    return binding.Fp8KVCache(s, batch, capacity, max(128, window), n_layers=1, device=DEV)


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    if case["op"] == "shared":
        return {"out": _plain_shared(st)}
    turn = _plain_turn(case, st["pos"])
    q = _plain_head(st["q"], st["gains"][0], case, turn).to(TYPES[case["out"]])
    k = _plain_head(st["k"], st["gains"][1], case, turn)
    if case["op"] == "rotate":
        return {"q": q, "k": k.to(TYPES[case["out"]])}
    return {"q": q, "k": list(k.to(torch.bfloat16)), "v": list(st["v"].to(torch.bfloat16))}


def _run_own(case, st):
    from paper_2608_10362_amd import binding
    if case["op"] == "shared":
        binding.specdec_attention_shared(st["prefix"], st["kv"], 0, st["q"], st["out"], workspace=st["ws"])
        return {"out": st["out"]}
    if case["op"] == "rotate":
        binding.specdec_rope_apply(st["rope"], st["q"], st["k"], st["q_out"], st["k_out"], positions=st["pos"])
        return {"q": st["q_out"], "k": st["k_out"]}
    binding.specdec_rope_append(st["kv"], 0, st["rope"], st["q"], st["k"], st["v"], st["q_out"])
    rows = [st["kv"].read_context(0, b, start, case["rows"]) for b, start in enumerate(st["starts"])]
    return {"q": st["q_out"], "k": [k for k, _ in rows], "v": [v for _, v in rows]}


def _plain_turn(case, pos):
    """Cosines and sines [B, n, 1, rotary / 2] of every pair's angle."""
    j = torch.arange(case["rotary"] // 2, dtype=torch.float64, device=DEV)
    angle = pos.double()[:, :, None, None] * torch.pow(torch.full_like(j, BASE), -2.0 * j / case["rotary"])
    return torch.cos(angle).float(), torch.sin(angle).float()


def _plain_head(x, gain, case, turn):
    """[B, n, heads, hd] -> the same, normalised and rotated, in 32 bits."""
    x = x.float()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    r, (cos, sin) = case["rotary"], turn
    y, rest = x[..., :r], x[..., r:]
    a, b = (y[..., 0::2], y[..., 1::2]) if case["interleaved"] else (y[..., :r // 2], y[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([y, rest], -1)


def _plain_shared(st):
    q, n_len = st["q"].float(), st["len"].long()
    B, n, H, hd = q.shape
    G, cap, tail = st["kc"].shape[2], st["kc"].shape[1], st["kt"].shape[1]
    r, P = H // G, st["case"]["prefix"]
    whole = P // BLOCK * BLOCK
    pk = torch.cat([_dequantize(st["pkc"], st["pks"])[:whole], st["pkt"].float()])  # the prefix: seen by every row
    pv = torch.cat([_dequantize(st["pvc"], st["pvs"])[:whole], st["pvt"].float()])
    scale = 1.0 / math.sqrt(hd)
    qs = q.reshape(B, n, G, r, hd).permute(2, 0, 1, 3, 4).reshape(G, B * n * r, hd)
    sp = torch.matmul(qs, pk.permute(1, 2, 0).contiguous()) * scale  # [G, B n r, P]
    sealed = n_len // BLOCK * BLOCK
    k = torch.cat([_dequantize(st["kc"], st["ks"]), st["kt"].float()], 1)
    v = torch.cat([_dequantize(st["vc"], st["vs"]), st["vt"].float()], 1)
    # positions of the own keys: a code counts below the last whole block's end, a tail row at its place
    i, j = torch.arange(cap, device=q.device)[None], torch.arange(tail, device=q.device)[None]
    far = torch.full((), 1 << 40, device=q.device)
    pos = torch.cat([torch.where(i < sealed[:, None], i, far), sealed[:, None] + j], 1)
    seen = pos[:, None] <= (n_len[:, None] + torch.arange(n, device=q.device))[:, :, None]  # [B, n, keys]
    qo = qs.reshape(G, B, n * r, hd).transpose(0, 1).contiguous()
    so = torch.matmul(qo, k.permute(0, 2, 3, 1).contiguous()) * scale  # [B, G, n r, keys]
    so = so.reshape(B, G, n, r, -1).masked_fill(~seen[:, None, :, None], -math.inf).reshape(B, G, n * r, -1)
    sp = sp.reshape(G, B, n * r, P).transpose(0, 1)
    m = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    ep, eo = torch.exp(sp - m), torch.exp(so - m)
    op = torch.matmul(ep.transpose(0, 1).reshape(G, B * n * r, P), pv.transpose(0, 1).contiguous())
    op = op.reshape(G, B, n * r, hd).transpose(0, 1)
    o = (op + torch.matmul(eo, v.transpose(1, 2).contiguous())) / (ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True))
    return o.reshape(B, G, n, r, hd).permute(0, 2, 1, 3, 4).reshape(B, n, H, hd).to(st["q"].dtype).contiguous()


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    H, G, hd, _ = SHAPES[case["shape"]]
    size = {"f32": 4.0, "bf16": 2.0}
    if case["op"] != "shared":
        rows = float(case["batch"]) * case["rows"]
        heads = H + G if case["op"] == "rotate" else H + 2 * G
        out = (H + G) * size[case["out"]] if case["op"] == "rotate" else H * size[case["out"]] + 2 * G * 2.0
        # (append: the rows written into the cache, and read back out of it)
        back = 0.0 if case["op"] == "rotate" else 2 * G * 2.0 * 2
        return {"bytes": rows * hd * (heads * size[case["dtype"]] + out + back),
                "flops": rows * (H + G) * hd * (7.0 if case["norm"] else 3.0)}
    n, P, B = case["new"], case["prefix"], case["batch"]
    whole = P // BLOCK * BLOCK
    nbytes, pairs = 2.0 * G * hd * (whole + 2.0 * (P - whole)), float(B) * n * P
    for L in _lengths(case):
        sealed = L // BLOCK * BLOCK
        nbytes += 2.0 * G * hd * (sealed + 2.0 * (L + n - sealed)) + 2 * size[case["dtype"]] * n * H * hd
        pairs += n * L + n * (n + 1) / 2
    return {"bytes": nbytes, "flops": 4.0 * H * hd * pairs}


# ---------------------------------------------------------------- 64-bit results
def _e4m3(x):
    """Nearest e4m3 value of |x| <= 448 (float64), ties to even: 3 mantissa bits, smallest exponent -6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_blocks(x, n):
    """The first n of [.., G, hd] bfloat16 rows, as a cache of n committed rows holds them, in 64 bits."""
    x = x.double()
    whole = n // BLOCK * BLOCK
    xb = x[:whole].reshape(whole // BLOCK, BLOCK, *x.shape[1:])
    amax = xb.abs().amax(dim=(1, 3), keepdim=True).clamp(min=2.0 ** -140)
    s = torch.exp2(torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(min=MIN_EXP))
    return torch.cat([(_e4m3(xb / s) * s).reshape(whole, *x.shape[1:]), x[whole:]])


def _exact_head(x, gain, case):
    """Norm, then each pair (a, b) as a + ib times e^(i angle)."""
    x = x.double()
    if gain is not None:
        x = gain.double() * x * (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).rsqrt()
    r = case["rotary"]
    half = r // 2
    at = torch.arange(half, device=DEV)
    first, second = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + half)
    pos = (torch.tensor(_starts(case), device=DEV, dtype=torch.float64)[:, None] +
           torch.arange(case["rows"], device=DEV, dtype=torch.float64))
    angle = pos[:, :, None, None] * torch.exp(at.double() * (-2.0 * math.log(BASE) / r))
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    H, G, hd, d = SHAPES[case["shape"]]
    B = case["batch"]
    if case["op"] != "shared":
        (q, k, v), (gq, gk) = _projections(case, seed), _gains(case, seed)
        q, k, v = _exact_head(q, gq, case), _exact_head(k, gk, case), v.double()
        return {"q": q, "k": k} if case["op"] == "rotate" else {"q": q, "k": list(k), "v": list(v)}
    n, P, lens, r = case["new"], case["prefix"], _lengths(case), H // G
    (pk, pv), (k, v) = _prefix_rows(case, seed), _own_rows(case, seed)
    q = _normal(seed, 31, (B, n, H, hd), 1.0, TYPES[case["dtype"]]).double()
    pk, pv = _exact_blocks(pk, P)[:P], _exact_blocks(pv, P)[:P]
    out = torch.empty((B, n, H, hd), dtype=torch.float64, device=DEV)
    for b in range(B):
        m = lens[b] + n
        kb = torch.cat([pk, _exact_blocks(k[b], lens[b])[:m]]).transpose(0, 1).contiguous()  # [G, P + m, hd]
        vb = torch.cat([pv, _exact_blocks(v[b], lens[b])[:m]]).transpose(0, 1).contiguous()
        late = torch.arange(P + m, device=DEV)[None] > P + lens[b] + torch.arange(n, device=DEV)[:, None]
        qb = q[b].reshape(n, G, r, hd).permute(1, 2, 0, 3).reshape(G, r * n, hd)
        s = torch.matmul(qb, kb.transpose(1, 2).contiguous()) / math.sqrt(hd)
        p = torch.softmax(s.reshape(G, r, n, -1).masked_fill(late, -math.inf), -1).reshape(G, r * n, -1)
        out[b] = torch.matmul(p, vb).reshape(G, r, n, hd).permute(2, 0, 1, 3).reshape(n, H, hd)
    return {"out": out}
