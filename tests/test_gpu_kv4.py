"""q4nx_kv_store, q4nx_kv4_load and q4nx_kv4_attention against the float64 oracle.

Tolerances (derived, none fitted):
  queries   a bf16 rounding, 2^-8 |o|; the float32 norm, (d + 8) 2^-24 relative (d squares summed one after another at
            worst); sine and cosine, SIN absolute each (measured over all turns by test_sine_and_cosine), and the few
            roundings of the rotation, together (SIN + (d + 16) 2^-24) (|lo| + |hi|).
  keys      half a step of the row's group, stretched and shifted by the bf16 roundings of scale and offset, plus the
            value's own rounding and the query's float32 terms: see _key_bound.
  values, and keys that are neither normed nor rotated: the bytes themselves.
  attention with u = 2^-24: a score is off by at most d u sum|q k| scale + 4 u |s|, so a weight by e = 2 x that (itself and
            the sum) + 2^-20 (exponentials, corrections); the sums over n positions add (n + 64) u; the weights' rounding
            2^-24 for a float32 output; for a bf16 one 2^-16 (two bf16 terms), or 2^-8 with many rows over a long range
            (one term: half a step of bf16, as the output's own rounding): e' sum p|v|.  Then the output's rounding.
"""
import numpy as np
import pytest

import oracle
from oracle import kv4

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SIN = 2.0 ** -18


@pytest.fixture(scope="module")
def q4():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_06063_amd as mod
    return mod


def _bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _freq(d, theta=1e4, div=1.0):
    return (theta ** (-np.arange(0, d, 2) / d) / div).astype(np.float32)


def _inputs(rng, T, width, f32):
    x = (2 * rng.standard_normal((T, width))).astype(np.float32)
    if f32:
        return x, torch.from_numpy(x).cuda()
    b = oracle.f32_to_bf16(x)
    return oracle.bf16_to_f32(b), _bf16(b)


def _rotated_tol(ref, d):
    h = d // 2
    mag = np.abs(ref[..., :h]) + np.abs(ref[..., h:])          # the pair's |lo| + |hi|: at least its length
    mag = np.concatenate([mag, mag], -1) * 1.5                 # (before the turn: at most sqrt 2 of it)
    return (SIN + (d + 16) * U) * mag + 1e-30


# ---- the store ------------------------------------------------------------------------------------------------------
# Every head dimension, types in and out, waves that mix queries, keys and values, heads that do not fill a wave,
# batches with padded places, one token and many (a wave of many heads), far positions.
STORE = [
    # H, G, d, B, T, L, f32, format, norm, rotation
    (32, 16, 128, 1, 1, 131072, False, 1, True, True),
    (8, 4, 256, 1, 1, 64, True, 1, True, True),
    (4, 1, 256, 5, 5, 40, False, 1, True, True),
    (3, 1, 64, 1, 77, 100, False, 1, True, True),
    (5, 3, 64, 4, 4, 33, True, 1, True, False),
    (1, 1, 128, 1, 33, 33, True, 1, False, True),
    (12, 4, 64, 1, 700, 2048, False, 1, True, True),
    (32, 16, 128, 1, 1500, 1600, True, 1, True, True),
    (8, 4, 256, 1, 1, 64, True, 0, True, True),
    (4, 1, 256, 33, 33, 1000, True, 0, True, True),
    (32, 16, 128, 1, 300, 333, False, 0, True, True),
    (7, 5, 64, 2, 2, 10, False, 0, False, False),
]


def _key_bound(ref, tol):
    g = ref.reshape(*ref.shape[:-1], -1, 32)
    lo, hi = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
    step = (hi - lo) / 15
    t = tol.reshape(g.shape)
    b = step * 0.5 * (1 + 2.0 ** -7) + 2.0 ** -8 * (np.abs(lo) + 15 * step) + 2.0 ** -8 * (np.abs(g) + step) + 3 * t.max(-1, keepdims=True)
    return b.reshape(ref.shape)


@pytest.mark.parametrize("H,G,d,B,T,L,f32,fmt,norm,rot", STORE)
def test_store(q4, H, G, d, B, T, L, f32, fmt, norm, rot):
    print("[case] store", H, G, d, B, T, L, f32, fmt, norm, rot, flush=True)
    rng = np.random.default_rng(H * 1000 + T)
    xh, x = _inputs(rng, T, (H + 2 * G) * d, f32)
    qw, kw = (oracle.f32_to_bf16(0.3 * rng.standard_normal(d).astype(np.float32)) for _ in range(2))
    f = _freq(d, 1e6, 8.0)
    if B == 1:
        pos = (L - T + np.arange(T)).astype(np.int32)
        seqs = None
        if T > 8:
            pos[3], pos[5] = -1, L + 7                                    # padding inside a chunk
    else:
        pos, seqs = rng.integers(0, L, T).astype(np.int32), rng.permutation(B)[:T].astype(np.int32)
        pos[0] = L - 1
        seqs[-1] = B                                                      # a sequence that is none: padding
    sv = np.zeros(T, np.int32) if seqs is None else seqs
    there = (pos >= 0) & (pos < L) & (sv < B)
    q_out = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    if fmt:
        before = rng.integers(0, 256, q4.q4nx_kv4_cache_size(B, G, d, L)).astype(np.uint8) if L < 4096 else np.zeros(
            q4.q4nx_kv4_cache_size(B, G, d, L), np.uint8)
        caches = [torch.from_numpy(before.copy()).cuda() for _ in range(2)]
    else:
        caches = [torch.full((B, G, L, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q4.q4nx_kv_store(x[:, :H * d], x[:, H * d:(H + G) * d], x[:, (H + G) * d:], _ints(pos), q_out, *caches, T, H, G, d, B, L,
                     fmt, seqs=None if seqs is None else _ints(seqs), q_weight=_bf16(qw) if norm else None,
                     k_weight=_bf16(kw) if norm else None, weight_offset=1.0, eps=1e-6,
                     inv_freq=torch.from_numpy(f).cuda() if rot else None)
    torch.cuda.synchronize()
    xh = xh.reshape(T, H + 2 * G, d)
    turned = [kv4.normed_rotated(part, w if norm else None, 1.0, 1e-6, pos, f if rot else None)
              for part, w in ((xh[:, :H], qw), (xh[:, H:H + G], kw))]
    got = q_out.float().cpu().numpy().astype(np.float64)
    tol = _rotated_tol(turned[0], d) + 2.0 ** -8 * np.abs(turned[0])
    assert (np.abs(got - turned[0]) <= tol)[there].all(), float((np.abs(got - turned[0]) / tol)[there].max())
    assert (got[~there] == 7.0).all()

    heads = (sv[:, None] * G + np.arange(G))[there].ravel()
    at = np.repeat(pos[there], G)
    kref, vrows = turned[1][there], np.ascontiguousarray(xh[:, H + G:][there])
    if not fmt:
        for c, ref in zip(caches, (kref, vrows.astype(np.float64))):
            got = c.float().cpu().numpy().astype(np.float64).reshape(B * G, L, d)
            new = got[heads, at].reshape(ref.shape)
            assert (np.abs(new - ref) <= _rotated_tol(ref, d) + 2.0 ** -8 * np.abs(ref)).all()
            got[heads, at] = 5.0
            assert (got == 5.0).all()                                     # every other row as it was
        return
    want = before.copy()
    kv4.write_rows(want, vrows.reshape(-1, d), heads, at, B * G, L, kv4.v_address)
    assert np.array_equal(caches[1].cpu().numpy(), want)
    k = caches[0].cpu().numpy()
    values = oracle.bf16_to_f32(kv4.read_rows(k, heads, at, B * G, L, d, kv4.k_address)).astype(np.float64).reshape(kref.shape)
    tol = _key_bound(kref, _rotated_tol(kref, d))
    assert (np.abs(values - kref) <= tol).all(), float((np.abs(values - kref) / tol).max())
    probe = np.arange(G * d, dtype=np.float32).reshape(G, d)              # the bytes of K's own rows, whatever they hold
    a, b = before.copy(), k.copy()
    for buf in (a, b):
        kv4.write_rows(buf, np.tile(probe, (len(at) // G, 1)), heads, at, B * G, L, kv4.k_address)
    assert np.array_equal(a, b)                                           # every other row as it was


def test_sine_and_cosine(q4):
    """All of a turn through a stored query: x = (1, 0) pairs with one frequency, so that q_out's halves are cosine and
    sine of positions * f; the pairs' values are read back in bf16, so this bounds SIN only to 2^-9; the float32 bound
    comes from scale: x = 1 and the other half 1, where lo = cos - sin vanishes at an eighth of a turn."""
    print("[case] sine and cosine", flush=True)
    T, d = 4096, 64
    f = np.full(d // 2, 2 * np.pi / 8, np.float32)                        # position p: p eighths of a turn, almost
    x = np.ones((T, 3 * d), np.float32)
    xd = torch.from_numpy(x).cuda()
    pos = np.arange(T, dtype=np.int32) * 1000 + 1
    q = torch.zeros(T, 1, d, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.zeros(1, 1, 4200000, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q4.q4nx_kv_store(xd[:, :d], xd[:, d:2 * d], xd[:, 2 * d:], _ints(pos), q, kc, vc, T, 1, 1, d, 1, 4200000, q4.Q4NX_KV_BF16,
                     inv_freq=torch.from_numpy(f).cuda())
    ref = kv4.normed_rotated(x[:, None, :d], None, 0, 0, pos, f)
    got = q.float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * SIN + 8 * U).all()
    assert (np.abs(ref) < 2.0 ** -8).any()                                # differences that only SIN bounds


def _hard_rows(rng, n, d):
    """Rows whose codes are hard to get right: ties, constants, signed zeros, tiny, huge, NaN and infinite values."""
    rows = rng.standard_normal((n, d)).astype(np.float32)
    rows[0] = 0.0
    rows[1] = -0.0
    rows[2] = 1.25
    rows[3] = (np.arange(d) % 31) * 0.5                                   # halves of a step
    rows[4, ::3] = np.nan
    rows[5, 1], rows[5, 40] = np.inf, -np.inf
    rows[6] *= 1e-32
    rows[7] = 1000.0 + rng.standard_normal(d).astype(np.float32) * 1e-4   # steps near the rounding of the offset
    rows[8] *= np.float32(1e38)
    rows[9] = -1.0
    rows[9, 17] = 2.0 ** 24
    return rows


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("fmt_f32", [True, False])
def test_codes_are_the_quantizers(q4, d, fmt_f32):
    print("[case] codes", d, fmt_f32, flush=True)
    rng = np.random.default_rng(d)
    G, T, L = 2, 24, 50
    rows = _hard_rows(rng, 2 * T * G, d)
    if not fmt_f32:
        rows = oracle.bf16_to_f32(oracle.f32_to_bf16(rows))
    k, v = rows[:T * G].reshape(T, G * d), rows[T * G:].reshape(T, G * d)
    v[:5 * 1] = k[:5]                                                     # the hard ones for V too
    dev = (lambda a: torch.from_numpy(a.copy()).cuda()) if fmt_f32 else (lambda a: _bf16(oracle.f32_to_bf16(a)))
    pos = rng.permutation(L)[:T].astype(np.int32)
    size = q4.q4nx_kv4_cache_size(1, G, d, L)
    caches = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    q = torch.zeros(T, 2 * d, dtype=torch.float32 if fmt_f32 else torch.bfloat16, device="cuda")
    q_out = torch.empty(T, 2, d, dtype=torch.bfloat16, device="cuda")
    q4.q4nx_kv_store(q, dev(k), dev(v), _ints(pos), q_out, *caches, T, 2, G, d, 1, L)
    heads, at = np.tile(np.arange(G), T), np.repeat(pos, G)
    for c, x, address in ((caches[0], k, kv4.k_address), (caches[1], v, kv4.v_address)):
        want = np.zeros(size, np.uint8)
        kv4.write_rows(want, x.reshape(-1, d), heads, at, G, L, address)
        assert np.array_equal(c.cpu().numpy(), want), address.__name__
    # and the reader, to both types; padding is left alone
    for dt in (torch.float32, torch.bfloat16):
        ask = np.concatenate([pos, [-1, L]]).astype(np.int32)
        out = [torch.full((T + 2, G, d), 3.0, dtype=dt, device="cuda") for _ in range(2)]
        q4.q4nx_kv4_load(*caches, _ints(ask), *out, T + 2, G, d, 1, L)
        for o, c, address in ((out[0], caches[0], kv4.k_address), (out[1], caches[1], kv4.v_address)):
            want = oracle.bf16_to_f32(kv4.read_rows(c.cpu().numpy(), heads, at, G, L, d, address)).reshape(T, G, d)
            got = o.float().cpu().numpy()
            assert np.array_equal(got[:T], want) and (got[T:] == 3.0).all()


def test_store_in_place_and_strided(q4):
    print("[case] store in place", flush=True)
    rng = np.random.default_rng(5)
    T, H, G, d, L = 50, 8, 4, 128, 64
    xh, x = _inputs(rng, T, (H + 2 * G) * d + 64, False)                  # rows longer than what they hold
    f = torch.from_numpy(_freq(d)).cuda()
    size = q4.q4nx_kv4_cache_size(1, G, d, L)
    out = []
    for inplace in (False, True):
        q = x[:, :H * d].contiguous() if inplace else x[:, :H * d]
        q_out = q if inplace else torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda")
        caches = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
        q4.q4nx_kv_store(q, x[:, H * d:(H + G) * d], x[:, (H + G) * d:(H + 2 * G) * d], _ints(np.arange(T)), q_out, *caches,
                         T, H, G, d, 1, L, inv_freq=f)
        out.append([_bits(q_out).reshape(T, -1)] + [c.cpu().numpy() for c in caches])
    assert all(np.array_equal(a, b) for a, b in zip(*out))


# ---- attention --------------------------------------------------------------------------------------------------------
def _cache(rng, q4, B, G, d, L, lens, garbage=True):
    """Quantized caches of sequences of lens positions and their values (bf16 bits [B][G][max][d]); bytes of rows that
    nobody stored are garbage, NaN and infinite scales among it."""
    P = kv4.padded(L)
    size = q4.q4nx_kv4_cache_size(B, G, d, L)
    out, values = [], []
    for address in (kv4.k_address, kv4.v_address):
        c = rng.integers(0, 256, size).astype(np.uint8)
        if garbage:
            c[B * G * P * d // 2:].view(np.uint16)[:] = rng.choice(np.array([0x7FC0, 0x7F80, 0xFF80, 0x7F7F], np.uint16),
                                                                   B * G * P * d // 16)
        vals = np.zeros((B, G, max(max(lens), 1), d), np.uint16)
        for b in range(B):
            for g in range(G):
                if lens[b]:
                    rows = rng.standard_normal((lens[b], d)).astype(np.float32) * np.exp(0.5 * rng.standard_normal(d)).astype(np.float32)
                    h = np.full(lens[b], b * G + g)
                    kv4.write_rows(c, rows, h, np.arange(lens[b]), B * G, L, address)
                    vals[b, g, :lens[b]] = kv4.read_rows(c, h, np.arange(lens[b]), B * G, L, d, address)
        out.append(torch.from_numpy(c).cuda())
        values.append(vals)
    return out, values


def _tiled(B, T, H, G, d, L, window):
    """Whether a call expands K and V and works in tiles of many rows."""
    rows, span = T * H // G, min(L, window + min(T, 16)) if window else L
    blocks = -(-span // 32) + (window > 0)
    return rows >= 192 and B * G * -(-rows // 16) * blocks > (20480 if d == 256 else 32768)


def _long(B, T, H, G, d):
    """A capacity from which on such a call does."""
    return 32 * (33000 // (B * G * -(-T * H // G // 16)) + 1)


def _check_attention(q4, H, G, d, lens, T, window, bf16, L=None, scale=None, seed=0, spread=1.5):
    print("[case] attention", H, G, d, lens, T, window, bf16, L, flush=True)
    rng = np.random.default_rng(seed + H + T)
    B = len(lens)
    L = L or max(max(lens), T, 1)
    scale = float(np.float32(scale or d ** -0.5))
    caches, (K, V) = _cache(rng, q4, B, G, d, L, lens)
    q = oracle.f32_to_bf16((spread * rng.standard_normal((B, T, H, d))).astype(np.float32))
    nbytes = q4.q4nx_kv4_workspace_size(B, T, H, G, d, L, window)
    work = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")   # NaNs
    o = torch.full((B, T, H, d), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    q4.q4nx_kv4_attention(_bf16(q), *caches, _ints(lens), B, T, H, G, d, L, window, scale, o, work if nbytes else None)
    first = o.clone()
    q4.q4nx_kv4_attention(_bf16(q), *caches, _ints(lens), B, T, H, G, d, L, window, scale, o, work if nbytes else None)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), o.view(torch.int16))
    got = o.float().cpu().numpy().astype(np.float64)
    worst = 0.0
    for b in range(B):
        ref, bound, dots = kv4.attention(q[b], K[b], V[b], lens[b], window, scale)
        ds = abs(scale) * dots * (d * U + 4 * U)
        rounding = 2.0 ** -24 if not bf16 else 2.0 ** -8 if _tiled(B, T, H, G, d, L, window) else 2.0 ** -16
        e = 2 * ds + 2.0 ** -20 + (lens[b] + 64) * U + rounding
        tol = e * bound + (2.0 ** -8 if bf16 else U) * np.abs(ref) + 1e-37
        err = np.abs(got[b] - ref)
        worst = max(worst, float((err / tol).max()))
        assert (err <= tol).all(), worst
    print("worst err/tol %.3f" % worst, flush=True)


# Lengths of one position, inside, at and past a block of 32, past a workgroup's and past several splits; every head
# dimension; groups of 1 to 16 query heads; sequences of unlike length, empty ones among them; rows of several tokens
# in one tile and in several; windows inside a block, across blocks and of one position.
@pytest.mark.parametrize("H,G,d,lens,T,window,bf16,L", [
    (4, 1, 256, [1], 1, 0, False, 1),
    (4, 1, 256, [31], 1, 0, False, 64),
    (8, 4, 256, [32], 1, 0, True, 32),
    (8, 4, 256, [33], 1, 0, False, 4096),
    (8, 4, 256, [129], 1, 0, False, 4096),
    (32, 16, 128, [1000], 1, 0, False, 1024),
    (32, 16, 128, [1000], 1, 0, True, 32768),
    (2, 2, 64, [777], 1, 0, False, 800),
    (5, 1, 64, [300], 1, 0, False, 300),
    (16, 1, 128, [515], 1, 0, False, 600),
    (7, 1, 256, [2049], 1, 0, True, 4100),
    (8, 4, 128, [700, 0, 33, 1], 1, 0, False, 700),
    (8, 4, 256, [500, 100, 0], 1, 64, True, 512),
    (4, 2, 64, [900], 1, 1, False, 900),
    (4, 2, 64, [900], 1, 37, False, 1000),
    (4, 2, 64, [900], 1, 5000, False, 900),
    (32, 16, 128, [205], 5, 0, False, 256),
    (8, 1, 64, [100, 3, 0], 5, 0, False, 128),
    (8, 2, 128, [64], 64, 0, False, 64),
    (6, 2, 64, [200], 77, 0, True, 201),
    (8, 4, 256, [150, 20], 50, 0, False, 150),
    (8, 4, 256, [150, 20], 50, 33, True, 150),
    (3, 1, 128, [300], 130, 17, False, 512),
    (16, 16, 64, [120], 120, 0, True, 120),
    (16, 1, 64, [90], 90, 40, False, 90),
    # many rows over short ranges, and in test_attention_tiles over long ones: tiles of 64 rows (two key parts) and, from 512 of 128 on, of 128; a
    # tile's last rows missing; a sequence shorter than its rows, and an empty one; windows that leave whole blocks of a
    # tile to some rows only
    (8, 4, 128, [333], 100, 0, False, 400),
    (8, 4, 256, [333], 333, 0, True, 333),
    (12, 4, 64, [700, 40, 0], 64, 0, False, 701),
    (4, 2, 64, [513], 257, 100, False, 600),
    (4, 2, 128, [513], 257, 1, True, 600),
    (16, 16, 64, [220], 220, 0, True, 220),
    (16, 1, 64, [90], 90, 40, False, 90),
    (6, 2, 256, [200], 90, 50, True, 201),
    (64, 64, 64, [250, 192, 5, 0], 192, 0, False, 260),
    (64, 64, 64, [250, 192, 5, 0], 192, 0, True, 260),
    (64, 64, 128, [250, 192, 5, 0], 192, 50, False, 260),
    (64, 64, 256, [300, 256, 5, 0], 256, 0, False, 300),
    (64, 64, 256, [300, 256, 5, 0], 256, 33, True, 300),
    # whole and ragged last splits, a sequence with one split beside one with several
    (4, 2, 128, [2100, 513, 40], 100, 0, False, 2200),
    (8, 1, 64, [1600], 27, 0, True, 4000),
    (4, 2, 256, [1057], 129, 0, False, 1057),
    (4, 2, 128, [1700, 900], 111, 1100, False, 2000),
    # rows with more splits than one wave merges at once
    (2, 1, 64, [20000], 1, 0, False, 20000),
])
def test_attention(q4, H, G, d, lens, T, window, bf16, L):
    _check_attention(q4, H, G, d, lens, T, window, bf16, L)


# Many rows over long ranges (L None: a capacity that makes it one, however short the sequences): the cases of many rows
# above, tiles whose range is split and not, windows inside a tile's range and across splits, on tiles of 64 rows and 128.
@pytest.mark.parametrize("H,G,d,lens,T,window,bf16,L", [
    (8, 4, 128, [333], 100, 0, False, None),
    (8, 4, 256, [333], 333, 0, True, None),
    (12, 4, 64, [700, 40, 0], 64, 0, False, None),
    (16, 16, 64, [220], 220, 0, True, None),
    (6, 2, 256, [2100], 90, 0, True, None),
    (64, 64, 64, [250, 192, 5, 0], 192, 0, False, 1000),
    (64, 64, 64, [250, 192, 5, 0], 192, 0, True, 1000),
    (64, 64, 128, [250, 192, 5, 0], 192, 0, False, 1000),
    (64, 64, 256, [300, 256, 5, 0], 256, 0, False, 300),
    (4, 2, 128, [2100, 513, 40], 100, 0, False, None),
    (8, 1, 64, [1600], 27, 0, True, None),
    (4, 2, 256, [1057], 129, 0, False, None),
    (32, 32, 128, [2000], 512, 1100, False, 2100),
    (32, 32, 64, [2000], 512, 1100, True, 2100),
    (100, 100, 64, [700], 512, 300, False, 800),
    (512, 512, 64, [300], 272, 50, False, 300),
    (700, 700, 64, [300], 272, 33, True, 300),
    (64, 64, 256, [700], 520, 280, True, 700),
    (20, 20, 128, [1500], 1500, 0, False, 1500),
])
def test_attention_tiles(q4, H, G, d, lens, T, window, bf16, L):
    L = L or max(_long(len(lens), T, H, G, d), max(lens))
    assert _tiled(len(lens), T, H, G, d, L, window)
    _check_attention(q4, H, G, d, lens, T, window, bf16, L)


def test_attention_tiles_peaked_and_flat(q4):
    L = _long(1, 110, 4, 2, 128)
    _check_attention(q4, 4, 2, 128, [400], 110, 0, False, L, scale=-0.3)
    _check_attention(q4, 4, 2, 128, [400], 110, 0, False, L, scale=1e-30)
    _check_attention(q4, 4, 2, 128, [400], 110, 0, False, L, spread=20.0)


def test_attention_peaked_and_flat(q4):
    _check_attention(q4, 4, 2, 128, [400], 1, 0, False, 400, spread=20.0)
    _check_attention(q4, 4, 2, 128, [400], 3, 0, False, 400, scale=-0.3)
    _check_attention(q4, 4, 2, 128, [400], 1, 0, False, 400, scale=1e-6)
    for T in (3, 110):                                                    # few rows and many
        _check_attention(q4, 4, 2, 128, [400], T, 0, False, 400, scale=-0.3)
        _check_attention(q4, 4, 2, 128, [400], T, 30, False, 400, scale=1e-30)
        _check_attention(q4, 4, 2, 128, [400], T, 0, False, 400, spread=20.0)


def test_attention_scale_zero_is_the_mean(q4):
    print("[case] scale 0", flush=True)
    rng = np.random.default_rng(4)
    H, G, d, n = 4, 2, 64, 130
    caches, (K, V) = _cache(rng, q4, 1, G, d, n, [n])
    for T in (2, 100):
        q = _bf16(oracle.f32_to_bf16(rng.standard_normal((1, T, H, d)).astype(np.float32)))
        o = torch.full((1, T, H, d), float("nan"), device="cuda")
        q4.q4nx_kv4_attention(q, *caches, _ints([n]), 1, T, H, G, d, n, 40, 0.0, o,
                              torch.empty(q4.q4nx_kv4_workspace_size(1, T, H, G, d, n, 40) + 16, dtype=torch.uint8, device="cuda"))
        v = oracle.bf16_to_f32(V[0]).astype(np.float64)
        ref = np.stack([v[:, max(0, p - 39):p + 1].mean(1) for p in range(n - T, n)])              # [T][G][d]
        assert np.allclose(o[0].cpu().numpy(), np.repeat(ref, H // G, 1), rtol=0, atol=6 * (n + 64) * U)


def test_attention_lengths_are_clamped(q4):
    """Lengths beyond the capacity and below zero are read as L and 0: reads stay inside the caches."""
    print("[case] clamped lengths", flush=True)
    rng = np.random.default_rng(8)
    H, G, d, L = 8, 4, 128, 96
    caches, _ = _cache(rng, q4, 2, G, d, L, [96, 96])
    q = _bf16(oracle.f32_to_bf16(rng.standard_normal((2, 1, H, d)).astype(np.float32)))
    out = []
    for lens in ([96, 0], [1 << 30, -5], [97, -2147483648]):
        o = torch.full((2, 1, H, d), float("nan"), device="cuda")
        q4.q4nx_kv4_attention(q, *caches, _ints(lens), 2, 1, H, G, d, L, 0, 0.1, o,
                              torch.empty(max(16, q4.q4nx_kv4_workspace_size(2, 1, H, G, d, L)), dtype=torch.uint8, device="cuda"))
        out.append(o)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2]) and not out[0][1].any() and torch.isfinite(out[0]).all()


def test_loaded_rows_give_flowkv_the_same_attention(q4):
    print("[case] against FlowKV on loaded rows", flush=True)
    rng = np.random.default_rng(9)
    H, G, d, n, L = 8, 4, 256, 3000, 4096
    gen = torch.Generator(device="cuda").manual_seed(3)
    kv = torch.randn(n, 2 * G * d, device="cuda", generator=gen)
    size = q4.q4nx_kv4_cache_size(1, G, d, L)
    caches = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pos = _ints(np.arange(n))
    q_all = torch.zeros(n, H * d, device="cuda")
    q4.q4nx_kv_store(q_all, kv[:, :G * d], kv[:, G * d:], pos, torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda"),
                     *caches, n, H, G, d, 1, L)
    rows = [torch.empty(n, G, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q4.q4nx_kv4_load(*caches, pos, *rows, n, G, d, 1, L)
    q = _bf16(oracle.f32_to_bf16(rng.standard_normal((H, d)).astype(np.float32)))
    flat = [r.permute(1, 0, 2).contiguous() for r in rows]
    for window in (0, 1024):
        a, b = torch.empty(H, d, device="cuda"), torch.empty(H, d, device="cuda")
        q4.q4nx_flowkv_decode(q, *flat, H, G, d, n, n - 1, window, 0.0625, a,
                              torch.empty(q4.q4nx_flowkv_workspace_size(H, d, n), dtype=torch.uint8, device="cuda"))
        q4.q4nx_kv4_attention(q, *caches, _ints([n]), 1, 1, H, G, d, L, window, 0.0625, b,
                              torch.empty(max(16, q4.q4nx_kv4_workspace_size(1, 1, H, G, d, L, window)), dtype=torch.uint8, device="cuda"))
        # both are within (n + d) 2^-24 of exact relative to sum p|v| <= 6 (values of 5 sigma and a quantizer step)
        assert (a - b).abs().max().item() <= 2 * 6 * ((n + d + 64) * U + 2.0 ** -20)


# ---- together: a prompt in two chunks, then tokens by a captured step whose positions and lengths move on -----------------
def test_prompt_and_captured_decode(q4):
    print("[case] prompt and captured decode", flush=True)
    from workloads import gen_weights
    rng = np.random.default_rng(11)
    H, G, d, D, L, window = 8, 4, 128, 512, 256, 0
    width = (H + 2 * G) * d
    codes, s, o_ = gen_weights(width, D, seed=3)
    blob = torch.from_numpy(q4.q4nx_pack(codes, s, o_)).cuda()
    qw, kw = (_bf16(oracle.f32_to_bf16(0.2 * rng.standard_normal(d).astype(np.float32))) for _ in range(2))
    f = torch.from_numpy(_freq(d)).cuda()
    size = q4.q4nx_kv4_cache_size(1, G, d, L)
    scale = d ** -0.5
    n_prompt, n_new = 150, 6
    X = _bf16(oracle.f32_to_bf16(rng.standard_normal((n_prompt + n_new, D)).astype(np.float32)))

    def layer(x, T, pos, lens, qkv, q, caches, o, work):
        q4.q4nx_gemm(T, width, D, x, blob, qkv)
        q4.q4nx_kv_store(qkv[:, :H * d], qkv[:, H * d:(H + G) * d], qkv[:, (H + G) * d:], pos, q, *caches, T, H, G, d, 1, L,
                         q_weight=qw, k_weight=kw, inv_freq=f)
        q4.q4nx_kv4_attention(q, *caches, lens, 1, T, H, G, d, L, window, scale, o, work)

    def buffers(T):
        return (torch.empty(T, width, device="cuda"), torch.empty(T, H, d, dtype=torch.bfloat16, device="cuda"))

    work = torch.empty(max(q4.q4nx_kv4_workspace_size(1, T, H, G, d, L) for T in (1, 50, 100)) + 16, dtype=torch.uint8, device="cuda")

    def prompt(caches):
        outs = []
        for a, b in ((0, 100), (100, 150)):
            T = b - a
            o = torch.empty(T, H, d, device="cuda")
            layer(X[a:b].contiguous(), T, _ints(np.arange(a, b)), _ints([b]), *buffers(T), caches, o, work)
            outs.append(o)
        return torch.cat(outs)

    def fresh():
        return [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        eager = fresh()
        whole = prompt(eager)
        steps = []
        for i in range(n_new):
            p = n_prompt + i
            o = torch.empty(1, H, d, device="cuda")
            layer(X[p:p + 1].contiguous(), 1, _ints([p]), _ints([p + 1]), *buffers(1), eager, o, work)
            steps.append(o)
        captured = fresh()
        prompt(captured)
        x, pos, lens, o = X[:1].clone(), _ints([n_prompt]), _ints([n_prompt + 1]), torch.empty(1, H, d, device="cuda")
        qkv, q = buffers(1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer(x, 1, pos, lens, qkv, q, captured, o, work)
        for i in range(n_new):
            p = n_prompt + i
            x.copy_(X[p:p + 1])
            pos.fill_(p)
            lens.fill_(p + 1)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, steps[i]), i
        assert torch.equal(eager[0], captured[0]) and torch.equal(eager[1], captured[1])

    # The outputs against float64 attention over the cache's own values and the library's own queries.
    heads = lambda n: (np.repeat(np.arange(G), n), np.tile(np.arange(n), G))  # noqa: E731
    n = n_prompt + n_new
    K, V = (kv4.read_rows(c.cpu().numpy(), *heads(n), G, L, d, a).reshape(G, n, d)
            for c, a in ((eager[0], kv4.k_address), (eager[1], kv4.v_address)))
    qkv, q = buffers(n)
    q4.q4nx_gemm(n, width, D, X, blob, qkv)
    scratch = fresh()
    q4.q4nx_kv_store(qkv[:, :H * d], qkv[:, H * d:(H + G) * d], qkv[:, (H + G) * d:], _ints(np.arange(n)), q, *scratch, n, H, G, d,
                     1, L, q_weight=qw, k_weight=kw, inv_freq=f)
    ref, bound, dots = kv4.attention(_bits(q), K, V, n, window, scale)
    got = torch.cat([whole] + steps).cpu().numpy().astype(np.float64)
    # A query of another batch may be off by a bf16 step (the projection's sums differ in order): 2^-8 of each product.
    ds = scale * dots * (2.0 ** -7 + (d + 4) * U)
    assert (np.abs(got - ref) <= (2 * ds + 2.0 ** -19 + (n + 64) * U) * bound).all()


def test_other_stream_and_small_workspace(q4):
    print("[case] another stream", flush=True)
    rng = np.random.default_rng(12)
    H, G, d, L = 8, 4, 128, 4096
    caches, _ = _cache(rng, q4, 1, G, d, L, [600])
    q = _bf16(oracle.f32_to_bf16(rng.standard_normal((1, 1, H, d)).astype(np.float32)))
    lens = _ints([600])
    need = q4.q4nx_kv4_workspace_size(1, 1, H, G, d, L)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    a, b = torch.empty(1, 1, H, d, device="cuda"), torch.empty(1, 1, H, d, device="cuda")
    q4.q4nx_kv4_attention(q, *caches, lens, 1, 1, H, G, d, L, 0, 0.1, a, work)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q4.q4nx_kv4_attention(q, *caches, lens, 1, 1, H, G, d, L, 0, 0.1, b, work, stream=s)
    s.synchronize()
    assert torch.equal(a, b)
    for bad in (work[:need - 1], None):
        with pytest.raises(q4.Q4NXError):
            q4.q4nx_kv4_attention(q, *caches, lens, 1, 1, H, G, d, L, 0, 0.1, b, bad)


def test_a_nan_query_stays_in_its_row(q4):
    """A row of NaN or infinity leaves the rows that share its tile, its blocks and its maximum's test alone."""
    print("[case] NaN query rows", flush=True)
    rng = np.random.default_rng(21)
    H, G, d, n = 8, 2, 128, 700
    L = _long(1, 60, H, G, d)
    assert _tiled(1, 60, H, G, d, L, 0)
    caches, _ = _cache(rng, q4, 1, G, d, L, [n])
    for T in (1, 5, 60):                                                  # one tile, two, and tiles of 64 rows
        q = _bf16(oracle.f32_to_bf16(rng.standard_normal((1, T, H, d)).astype(np.float32)))
        bad = q.clone()
        bad[0, T // 2, 1] = float("nan")
        bad[0, 0, 6, 3] = float("inf")
        work = torch.empty(max(16, q4.q4nx_kv4_workspace_size(1, T, H, G, d, L)), dtype=torch.uint8, device="cuda")
        o = [torch.empty(1, T, H, d, device="cuda") for _ in range(2)]
        for x, y in zip((q, bad), o):
            q4.q4nx_kv4_attention(x, *caches, _ints([n]), 1, T, H, G, d, L, 0, 0.1, y, work)
        assert torch.isnan(o[1][0, T // 2, 1]).all() and torch.isnan(o[1][0, 0, 6]).all() and torch.isfinite(o[0]).all()
        keep = torch.ones(T, H, dtype=torch.bool, device="cuda")
        keep[T // 2, 1] = keep[0, 6] = False
        # (a maximum that one row moves is moved for all 16 or 32 of them, so the roundings of the others may differ)
        tol = 4 * ((n + 64) * U + 2.0 ** -20) * 12                        # |v| < 12: 4 sigma, a spread of e^1, a step
        assert (o[1][0][keep] - o[0][0][keep]).abs().max().item() <= tol


def test_bf16_cache_is_flowkvs(q4):
    """A bf16 cache that the store has written, read by q4nx_flowkv_decode."""
    print("[case] bf16 cache and FlowKV", flush=True)
    rng = np.random.default_rng(22)
    H, G, d, n, L = 8, 4, 256, 130, 160
    xh, x = _inputs(rng, n, (H + 2 * G) * d, False)
    f = torch.from_numpy(_freq(d)).cuda()
    caches = [torch.full((G, L, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q = torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda")
    for a, b in ((0, 129), (129, 130)):
        q4.q4nx_kv_store(x[a:b, :H * d], x[a:b, H * d:(H + G) * d], x[a:b, (H + G) * d:], _ints(np.arange(a, b)), q[a:b], *caches,
                         b - a, H, G, d, 1, L, kv_format=q4.Q4NX_KV_BF16, inv_freq=f)
    o = torch.empty(H, d, device="cuda")
    q4.q4nx_flowkv_decode(q[n - 1], *caches, H, G, d, L, n - 1, 100, 0.0625, o,
                          torch.empty(q4.q4nx_flowkv_workspace_size(H, d, L), dtype=torch.uint8, device="cuda"))
    K, V = (_bits(c[:, :n]) for c in caches)
    ref, bound, dots = kv4.attention(_bits(q[n - 1:]), K, V, n, 100, 0.0625)
    tol = (2 * 0.0625 * dots * (d + 4) * U + 2.0 ** -20 + (n + d + 64) * U) * bound
    assert (np.abs(o.cpu().numpy().astype(np.float64) - ref[0]) <= tol[0]).all()
    assert torch.isnan(caches[0][:, n:]).all() and torch.isnan(caches[1][:, n:]).all()


def test_captured_prompt_and_two_streams(q4):
    """A call with many rows, captured: replays follow the lengths; two calls at once with a workspace each give what
    each gives alone."""
    print("[case] captured prompt, two streams", flush=True)
    rng = np.random.default_rng(23)
    H, G, d, L, T, B = 8, 2, 128, 17000, 64, 2
    assert _tiled(B, T, H, G, d, L, 0)
    caches, _ = _cache(rng, q4, B, G, d, L, [1500, 1500])
    q = _bf16(oracle.f32_to_bf16(rng.standard_normal((B, T, H, d)).astype(np.float32)))
    one = q[:, -1:].contiguous()
    nbytes = [q4.q4nx_kv4_workspace_size(B, t, H, G, d, L) for t in (T, 1)]
    assert min(nbytes) > 0

    def run(lens, o, work, stream=None):
        q4.q4nx_kv4_attention(q, *caches, lens, B, T, H, G, d, L, 0, 0.1, o[0], work[0], stream=stream)
        q4.q4nx_kv4_attention(one, *caches, lens, B, 1, H, G, d, L, 0, 0.1, o[1], work[1], stream=stream)

    def buffers():
        return ([torch.full((B, t, H, d), float("nan"), device="cuda") for t in (T, 1)],
                [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in nbytes])

    cases = [[1500, 3], [64, 1500], [0, 700], [1, 513]]
    want = []
    for lens in cases:
        o, work = buffers()
        run(_ints(lens), o, work)
        want.append(o)
    torch.cuda.synchronize()
    lens, (o, work) = _ints(cases[0]), buffers()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(lens, o, work)
    for case, w in zip(cases + cases, want + want):
        lens.copy_(_ints(case))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, w)), case
        run(_ints(case), *buffers())                                      # eager work between replays

    streams, sets, at = [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(2)], [_ints(c) for c in cases[:2]]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, (o, work), lens in zip(streams, sets, at):
            run(lens, o, work, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for (o, _), w in zip(sets, want) for a, b in zip(o, w))


def test_padded_batch(q4):
    """A step of a batch with a free slot: its token is padding, its length 0; its output is zero, its query untouched."""
    print("[case] a free slot in a batch", flush=True)
    rng = np.random.default_rng(24)
    H, G, d, L, B = 4, 1, 256, 64, 3
    xh, x = _inputs(rng, B, (H + 2 * G) * d, True)
    caches, _ = _cache(rng, q4, B, G, d, L, [9, 33, 20], garbage=False)
    before = [c.clone() for c in caches]
    q, o = torch.full((B, H, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, 1, H, d), float("nan"), device="cuda")
    q4.q4nx_kv_store(x[:, :H * d], x[:, H * d:(H + G) * d], x[:, (H + G) * d:], _ints([9, -1, 20]), q, *caches, B, H, G, d, B, L,
                     seqs=_ints([0, 1, 2]))
    q4.q4nx_kv4_attention(q, *caches, _ints([10, 0, 21]), B, 1, H, G, d, L, 0, 0.1, o)
    assert (q[1] == 7.0).all() and not o[1].any() and torch.isfinite(o).all() and o[0].any() and o[2].any()
    P = kv4.padded(L)
    for c, was in zip(caches, before):
        codes, old = c[:B * G * P * d // 2].view(B, -1), was[:B * G * P * d // 2].view(B, -1)
        assert torch.equal(codes[1], old[1]) and not torch.equal(codes[0], old[0])
