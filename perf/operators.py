"""What lies between the q/k/v projections and the output projection of a layer, with a cache held in 4 bits: the
norm of queries and keys for each head, the rotation and the cache write (q4nx_kv_store, with q4nx_kv4_load as the
reader of rows), and the attention over that cache (q4nx_kv4_attention), for single tokens, batches and prompts.

Kinds of case:
  store    T tokens' projections are normed, rotated and stored.  Into the 4-bit cache, the stored rows come back as
           the values they stand for; into the bf16 cache, the cache itself is the output.
  attend   T query rows of each of B sequences attend over the 4-bit cache, the T rows being the last T positions of
           their sequence.

Every size is from the Gemma3 models of workloads/ or generic.  Inputs are synthetic: normal projections, caches of
normal rows with channels of unlike strength, quantized here.

The 4-bit cache, for K or V: B * G heads of P = ceil(L / 32) * 32 positions of d values in groups of 32, first every
head's codes, then every head's (scale, offset) pairs, value = bf16(scale * code + offset).
  K codes   [head][position][d / 8][4 bytes]: byte b of word s holds value 8s + b (low nibble) and 8s + 4 + b.
  K pairs   [head][position][d / 32]
  V codes   [head][P / 32][d / 64][4 h][16 n][2 e][2 a][4 r]: the byte of position 32 blk + 16a + 4h + r holds the values
            64 pair + 32e + n (low nibble) and + 16.
  V pairs   [head][P / 32][d / 32][4 h][2 a][4 r]
"""
import math

import torch

own = False

HEADS = {"1b": (4, 1, 256), "4b": (8, 4, 256), "27b": (32, 16, 128)}  # query heads, KV heads, head dimension
WINDOW = 1024
EPS = 1e-6
WORK_BYTES = 256 << 20  # the program's one workspace, for every layer and call


def listed():
    return [
        # One token of the largest model, far into a long context: the smallest call, once a layer and token.
        {"name": "store 27b token", "kind": "store", "H": 32, "G": 16, "d": 128, "B": 1, "T": 1, "p0": 100003, "L": 131072, "format": "q4", "in": "bf16", "theta": 1e6, "div": 8.0},
        # A batch of decoding users, one of them a padded place; float32 projections, the bf16 cache of FlowKV.
        {"name": "store 1b batch bf16 cache", "kind": "store", "H": 4, "G": 1, "d": 256, "B": 33, "T": 33, "p0": 900, "L": 1000, "format": "bf16", "in": "f32", "theta": 1e4, "div": 1.0},
        # The chunks that long prompts are cut into.
        {"name": "store 4b chunk", "kind": "store", "H": 8, "G": 4, "d": 256, "B": 1, "T": 2048, "p0": 2048, "L": 4096, "format": "q4", "in": "f32", "theta": 1e4, "div": 1.0},
        {"name": "store 27b chunk", "kind": "store", "H": 32, "G": 16, "d": 128, "B": 1, "T": 4096, "p0": 0, "L": 4096, "format": "q4", "in": "bf16", "theta": 1e6, "div": 8.0},
        # One token at the start of an answer.
        {"name": "attend 1b short", "kind": "attend", "H": 4, "G": 1, "d": 256, "B": 1, "T": 1, "n": 100, "L": 512, "window": 0, "out": "bf16"},
        # One token of a sliding-window layer, and of a global layer with a long context.
        {"name": "attend 4b window", "kind": "attend", "H": 8, "G": 4, "d": 256, "B": 1, "T": 1, "n": 20011, "L": 32768, "window": 1024, "out": "f32"},
        {"name": "attend 27b 32k", "kind": "attend", "H": 32, "G": 16, "d": 128, "B": 1, "T": 1, "n": 32768, "L": 32768, "window": 0, "out": "bf16"},
        # A batch of decoding users with contexts of every length, one place empty.
        {"name": "attend 4b batch", "kind": "attend", "H": 8, "G": 4, "d": 256, "B": 16, "T": 1, "n": 8191, "L": 8192, "window": 0, "out": "bf16"},
        # A drafted continuation of five tokens checked at once.
        {"name": "attend 27b draft", "kind": "attend", "H": 32, "G": 16, "d": 128, "B": 3, "T": 5, "n": 5003, "L": 8192, "window": 0, "out": "f32"},
        # A prompt's first chunk, a ragged later chunk in a sliding-window layer, and the longest chunk of the benchmark.
        {"name": "prompt 4b chunk", "kind": "attend", "H": 8, "G": 4, "d": 256, "B": 1, "T": 2048, "n": 2048, "L": 2048, "window": 0, "out": "bf16"},
        {"name": "prompt 27b window", "kind": "attend", "H": 32, "G": 16, "d": 128, "B": 1, "T": 777, "n": 5001, "L": 8192, "window": 1024, "out": "f32"},
        {"name": "prompt 27b chunk", "kind": "attend", "H": 32, "G": 16, "d": 128, "B": 1, "T": 4096, "n": 8192, "L": 8192, "window": 0, "out": "bf16"},
    ]


def _spread(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    H, G, d = rng.choice(sorted(HEADS.values()) + [(8, 8, 64), (8, 1, 128), (12, 4, 64)])
    if rng.random() < 0.3:
        B = rng.choice([1, 1, _spread(rng, 2, 64)])
        T = B if B > 1 else _spread(rng, 1, 4096)
        p0 = _spread(rng, 1, 50000)
        L = p0 + T + rng.randint(0, 100) if B == 1 else min(p0, 2000) + rng.randint(1, 100)
        return {"kind": "store", "H": H, "G": G, "d": d, "B": B, "T": T, "p0": p0 if B == 1 else min(p0, 2000), "L": L, "format": rng.choice(["q4", "q4", "bf16"]) if L <= 4096 else "q4",
                "in": rng.choice(["f32", "bf16"]), "theta": rng.choice([1e4, 1e6]), "div": rng.choice([1.0, 8.0])}
    window, out = rng.choice([0, 0, WINDOW, _spread(rng, 1, 4096)]), rng.choice(["f32", "bf16", "bf16"])
    if rng.random() < 0.6:  # single tokens, or a few
        B, T = rng.choice([1, 1, _spread(rng, 2, 32)]), rng.choice([1, 1, _spread(rng, 2, 12)])
        n = _spread(rng, T, 65536 // B)
    else:
        B, T = rng.choice([1, 1, 2]), _spread(rng, 16, 2500)
        n = T + rng.choice([0, _spread(rng, 1, 4096)])
    return {"kind": "attend", "H": H, "G": G, "d": d, "B": B, "T": T, "n": n, "L": n + rng.randint(0, 70), "window": window, "out": out}


def _lengths(case):
    """The sequences' lengths: the first is the longest, the last of several is an empty place."""
    B, n = case["B"], case["n"]
    return [n * (B - 1 - b) // (B - 1) if B > 1 else n for b in range(B)]


def _positions(case):
    """The tokens' positions: one run of one sequence, or a token of each sequence, the last place of several padded."""
    B, T, p0 = case["B"], case["T"], case["p0"]
    return list(range(p0, p0 + T)) if B == 1 else [p0 - 7 * b if p0 >= 7 * b else 0 for b in range(T - 1)] + [-1]


# ---- the 4-bit cache in torch operations --------------------------------------------------------------------------
def _pairs_and_codes(x):
    """float32 [..., d] -> scales, offsets (bf16 [..., d / 32]) and codes (uint8 [..., d]), the nearest code of each."""
    g = torch.nan_to_num(x, nan=0.0, posinf=2.0 ** 100, neginf=-2.0 ** 100).clamp(-2.0 ** 100, 2.0 ** 100).unflatten(-1, (-1, 32))
    lo, hi = g.amin(-1) + 0.0, g.amax(-1)
    scale, offset = ((hi - lo) / 15.0).bfloat16(), lo.bfloat16()
    scale, offset = (torch.where(t.abs().float() < 2.0 ** -100, t * 0, t) for t in (scale, offset))
    s, o = scale.float().unsqueeze(-1), offset.float().unsqueeze(-1)
    near = torch.where(s != 0, (g - o) / torch.where(s != 0, s, torch.ones_like(s)), torch.zeros_like(g)).clamp(0, 15).round()

    def off(q):  # the distance of code q's value, in 64 bits
        return ((s * q + o).double() - g.double()).abs()

    low, high = (near - 1).clamp(min=0), (near + 1).clamp(max=15)
    code = torch.where(off(low) <= off(near), low, near)
    code = torch.where(off(high) < off(code), high, code)
    return scale, offset, code.to(torch.uint8).flatten(-2)


def _values(scale, offset, code):
    """What the codes stand for: bf16 of the float32 scale * code + offset."""
    v = scale.float().unsqueeze(-1) * code.unflatten(-1, (-1, 32)).float() + offset.float().unsqueeze(-1)
    return v.bfloat16().flatten(-2)


def _blob(codes, pairs):
    return torch.cat([codes.reshape(-1), pairs.contiguous().reshape(-1).view(torch.uint8)])


def _pack(x, transposed):
    """float32 [heads][P][d] -> the cache's bytes (`transposed`: V's order)."""
    scale, offset, code = _pairs_and_codes(x)
    pairs = torch.stack([scale, offset], -1)
    if not transposed:
        c = code.unflatten(-1, (-1, 2, 4))
        return _blob(c[..., 0, :] | (c[..., 1, :] << 4), pairs)
    heads, P, d = x.shape
    c = code.view(heads, P // 32, 2, 4, 4, d // 64, 2, 2, 16)                # blk a h r pair e nibble n
    c = c[..., 0, :] | (c[..., 1, :] << 4)                                   # blk a h r pair e n
    p = pairs.view(heads, P // 32, 2, 4, 4, d // 32, 2)                      # blk a h r group
    return _blob(c.permute(0, 1, 5, 3, 7, 6, 2, 4).contiguous(), p.permute(0, 1, 5, 3, 2, 4, 6))


def _unpack(blob, heads, P, d, transposed):
    """The cache's bytes -> its values, bf16 [heads][P][d]."""
    n = heads * P * d // 2
    codes, pairs = blob[:n], blob[n:].view(torch.bfloat16)
    if transposed:
        codes = codes.view(heads, P // 32, d // 64, 4, 16, 2, 2, 4).permute(0, 1, 6, 3, 7, 2, 5, 4)   # blk a h r pair e n
        code = torch.stack([codes & 15, codes >> 4], -2).reshape(heads, P, d)
        pairs = pairs.view(heads, P // 32, d // 32, 4, 2, 4, 2).permute(0, 1, 4, 3, 5, 2, 6).reshape(heads, P, d // 32, 2)
    else:
        codes = codes.view(heads, P, d // 8, 1, 4)
        code = torch.cat([codes & 15, codes >> 4], -2).reshape(heads, P, d)
        pairs = pairs.view(heads, P, d // 32, 2)
    return _values(pairs[..., 0], pairs[..., 1], code)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def prepare(case, seed):
    gen = _gen(seed)
    H, G, d, B, T, L = (case[k] for k in ("H", "G", "d", "B", "T", "L"))
    P = -(-L // 32) * 32
    state = dict(case, P=P, work=torch.empty(WORK_BYTES, dtype=torch.uint8, device="cuda"))
    if case["kind"] == "store":
        dt = torch.float32 if case["in"] == "f32" else torch.bfloat16
        state["qkv"] = (2.0 * _randn(gen, T, (H + 2 * G) * d)).to(dt)        # one stacked projection's output
        state["q_weight"], state["k_weight"] = ((0.2 * _randn(gen, d)).bfloat16() for _ in range(2))
        f = case["theta"] ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d) / case["div"]
        state["inv_freq"] = f.float()
        state["positions"] = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
        state["seqs"] = torch.arange(T, dtype=torch.int32, device="cuda") if B > 1 else None
        state["q_out"] = torch.zeros(T, H, d, dtype=torch.bfloat16, device="cuda")
        if case["format"] == "q4":
            state["k_cache"], state["v_cache"] = (torch.zeros(B * G * P * d * 5 // 8, dtype=torch.uint8, device="cuda") for _ in range(2))
            state["k_rows"], state["v_rows"] = (torch.zeros(T, G, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        else:
            state["k_cache"], state["v_cache"] = (torch.zeros(B, G, L, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return state
    strength = torch.exp(0.5 * _randn(gen, 2, B * G, 1, d))                  # channels of unlike strength
    k = _randn(gen, B * G, P, d) * strength[0]
    state["k_cache"] = _pack(k, False)
    state["v_cache"] = _pack(_randn(gen, B * G, P, d) * strength[1], True)
    del k
    state["q"] = (1.5 * _randn(gen, B, T, H, d)).bfloat16()
    state["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    state["scale"] = d ** -0.5
    state["o"] = torch.zeros(B, T, H, d, dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(s):
    return _store(s) if s["kind"] == "store" else _attend(s)


def _store(s):
    H, G, d, B, T, L = (s[k] for k in ("H", "G", "d", "B", "T", "L"))
    q, k, v = s["qkv"][:, :H * d], s["qkv"][:, H * d:(H + G) * d], s["qkv"][:, (H + G) * d:]
    if own:
        import paper_2602_06063_amd as q4
        fmt = q4.Q4NX_KV_Q4 if s["format"] == "q4" else q4.Q4NX_KV_BF16
        q4.q4nx_kv_store(q, k, v, s["positions"], s["q_out"], s["k_cache"], s["v_cache"], T, H, G, d, B, L, fmt, seqs=s["seqs"],
                         q_weight=s["q_weight"], k_weight=s["k_weight"], weight_offset=1.0, eps=EPS, inv_freq=s["inv_freq"])
        if s["format"] == "bf16":
            return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}
        q4.q4nx_kv4_load(s["k_cache"], s["v_cache"], s["positions"], s["k_rows"], s["v_rows"], T, G, d, B, L, seqs=s["seqs"])
        return {"q": s["q_out"], "k": s["k_rows"], "v": s["v_rows"]}
    there = s["positions"] >= 0
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()        # far positions: in 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, w):
        x = x.float().unflatten(-1, (-1, d))
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * (1.0 + w.float())
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    keep = there[:, None, None]
    q, k, v = turned(q, s["q_weight"]), turned(k, s["k_weight"]), v.float().unflatten(-1, (-1, d))
    q = torch.where(keep, q.bfloat16(), s["q_out"])
    if s["format"] == "bf16":
        slot = s["positions"].clamp(min=0).long()
        seq = s["seqs"].long() if s["seqs"] is not None else torch.zeros_like(slot)
        for new, cache in ((k, s["k_cache"]), (v, s["v_cache"])):
            cache[seq, :, slot] = torch.where(keep, new.bfloat16(), cache[seq, :, slot])
        return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}
    return {"q": q, "k": torch.where(keep, _values(*_pairs_and_codes(k)), s["k_rows"]),
            "v": torch.where(keep, _values(*_pairs_and_codes(v)), s["v_rows"])}


def _attend(s):
    H, G, d, B, T, L, P, window = (s[k] for k in ("H", "G", "d", "B", "T", "L", "P", "window"))
    if own:
        import paper_2602_06063_amd as q4
        q4.q4nx_kv4_attention(s["q"], s["k_cache"], s["v_cache"], s["lens"], B, T, H, G, d, L, window, s["scale"], s["o"], s["work"])
        return s["o"]
    low, high = _range(s)                                                    # the positions that any row attends to
    k = _unpack(s["k_cache"], B * G, P, d, False)[:, low:high].float()
    v = _unpack(s["v_cache"], B * G, P, d, True)[:, low:high].float()
    q = s["q"].view(B, T, G, H // G, d).permute(0, 2, 1, 3, 4).reshape(B * G, T * (H // G), d).float()
    score = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
    row = s["lens"].view(B, 1) - T + torch.arange(T, device="cuda")          # each row's own position
    at = torch.arange(low, high, device="cuda")
    sees = (at <= row[..., None]) & ((at > row[..., None] - window) if window else (at >= 0))
    sees = sees.view(B, 1, T, 1, high - low)
    score = score.view(B, G, T, H // G, high - low).masked_fill(~sees, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B * G, -1, high - low), v).view(B, G, T, H // G, d)
    o = torch.where(total == 0, torch.zeros_like(o), o / total)
    return o.permute(0, 2, 1, 3, 4).reshape(B, T, H, d).to(s["o"].dtype)


def _range(case):
    high = max(_lengths(case))
    low = max(0, min(_lengths(case)) - case["T"] - case["window"] + 1) if case["window"] else 0
    return low, high


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    H, G, d, B, T = (case[k] for k in ("H", "G", "d", "B", "T"))
    if case["kind"] == "store":
        n, size = sum(p >= 0 for p in _positions(case)), 4 if case["in"] == "f32" else 2
        rows = 2 * G * d * (2 * 0.625 + 2 if case["format"] == "q4" else 2)  # written, read back and written out as values
        return {"bytes": n * ((H + 2 * G) * d * size + H * d * 2 + rows), "flops": n * 10.0 * (H + 2 * G) * d}
    pairs = read = 0
    for n in _lengths(case):
        first, window = max(0, n - T), case["window"] or n
        full = range(first, n)                                               # positions of the rows that there are
        if len(full):
            ramp = max(0, min(n, window) - first)                            # rows that see their whole past
            pairs += ramp * (first + 1 + first + ramp) // 2 + (len(full) - ramp) * window
            read += n - max(0, first - window + 1)
    size = 4 if case["out"] == "f32" else 2
    return {"bytes": read * 2 * G * d * 0.625 + B * T * H * d * (2 + size) + 4 * B, "flops": 4.0 * d * H * pairs}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    H, G, d, B, T, P = (s[k] for k in ("H", "G", "d", "B", "T", "P"))
    dev = "cuda"
    if case["kind"] == "store":
        x = s["qkv"].double().view(T, H + 2 * G, d)
        out = torch.zeros_like(x)
        half = d // 2
        turn = torch.exp(1j * (s["positions"].double()[:, None, None] * s["inv_freq"].double()))
        for first, count, w in ((0, H, s["q_weight"]), (H, G, s["k_weight"])):
            r = x[:, first:first + count]
            r = r / torch.sqrt(r.square().sum(-1, keepdim=True) / d + EPS) * (w.double() + 1)
            z = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * turn
            out[:, first:first + count] = torch.cat([z.real, z.imag], -1)
        out[:, H + G:] = x[:, H + G:]
        gone = (s["positions"] < 0)[:, None, None]
        out = out.masked_fill(gone, 0.0)
        if case["format"] == "bf16":
            k, v = (torch.zeros(B, G, case["L"], d, dtype=torch.float64, device=dev) for _ in range(2))
            for t, p in enumerate(_positions(case)):
                if p >= 0:
                    k[t if B > 1 else 0, :, p], v[t if B > 1 else 0, :, p] = out[t, H:H + G], out[t, H + G:]
            return {"q": out[:, :H], "k": k, "v": v}
        # A key's code is a decision between neighbours that the last bit of its rotation can turn: no value in 64 bits.
        return {"q": out[:, :H], "k": None, "v": _quantized(s["qkv"].float().view(T, H + 2 * G, d)[:, H + G:]).masked_fill(gone, 0.0)}
    lens, W = _lengths(case), case["window"] or case["n"] + 1
    o = torch.zeros(B, T, H, d, dtype=torch.float64, device=dev)
    if 4.0 * d * H * T * max(lens) * B > 4e12:
        return None
    n_codes = B * G * P * d // 2
    e = torch.arange(d, device=dev)
    for b in range(B):
        n = lens[b]
        rows = torch.arange(max(0, T - n), T, device=dev)
        if not len(rows):
            continue
        at = n - T + rows
        low = max(0, int(at[0]) - W + 1)
        j = torch.arange(low, n, device=dev)[:, None]
        for g in range(G):
            head = b * G + g
            # K: the byte and the nibble of value e of position j, one formula each
            byte = s["k_cache"][(head * P + j) * (d // 2) + (e // 8) * 4 + e % 4].to(torch.int64)
            code = torch.where(e % 8 >= 4, byte >> 4, byte & 15)
            k = _at(s["k_cache"], n_codes, (head * P + j) * (d // 32) + e // 32, code)
            blk, a, h, r = j // 32, j % 32 // 16, j % 16 // 4, j % 4
            pair, half, nib, m = e // 64, e % 64 // 32, e % 32 // 16, e % 16
            byte = s["v_cache"][head * P * (d // 2) + blk * 16 * d + pair * 1024 + (h * 16 + m) * 16 + half * 8 + a * 4 + r].to(torch.int64)
            code = torch.where(nib.expand_as(byte) == 1, byte >> 4, byte & 15)
            v = _at(s["v_cache"], n_codes, head * P * (d // 32) + blk * d + (e // 32) * 32 + h * 8 + a * 4 + r, code)
            for hq in range(g * (H // G), (g + 1) * (H // G)):
                score = s["q"][b, rows, hq].double() @ k.T * s["scale"]
                score[(j.T > at[:, None]) | (j.T <= at[:, None] - W)] = -math.inf
                o[b, rows, hq] = torch.softmax(score, -1) @ v
    return o


def _at(blob, first, pair, code):
    """Values of codes with the pair of each: float32 of the exact scale * code + offset, then bf16."""
    pairs = blob[first:].view(torch.bfloat16).double().view(-1, 2)[pair]
    return (pairs[..., 0] * code + pairs[..., 1]).float().bfloat16().double()


def _quantized(x):
    """The values that float32 rows are stored as: of all 16 values of a group's pair, the nearest, the lowest on a tie."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    lo, hi = g.min(-1).values, g.max(-1).values
    scale, offset = ((hi - lo) / 15).bfloat16().double()[..., None], lo.bfloat16().double()[..., None]
    best, found = None, None
    for c in range(16):
        value = (scale * c + offset).float().double()
        far = (value - g.double()).abs()
        best, found = (far, value.expand_as(far)) if c == 0 else (torch.minimum(best, far), torch.where(far < best, value, found))
    return found.float().bfloat16().double().reshape(x.shape)
