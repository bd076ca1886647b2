"""q4nx_kv_store, q4nx_kv4_load and q4nx_kv4_attention on the host: sizes, and every refusal, which all come before any
HIP call (no GPU here: device entry points are only called with invalid arguments)."""
import ctypes

import pytest

import paper_2602_06063_amd as q4

A = 1 << 20          # aligned, never dereferenced
LIB = q4.lib


def test_sizes():
    size, work = LIB.q4nx_kv4_cache_size, LIB.q4nx_kv4_workspace_size
    for B, G, d, L in [(1, 1, 64, 1), (1, 16, 128, 32), (3, 4, 256, 33), (2, 5, 64, 1000), (1, 16, 128, 1 << 30)]:
        assert size(B, G, d, L) == B * G * -(-L // 32) * 32 * d * 5 // 8 == q4._cache_bytes(B, G, d, L, q4.Q4NX_KV_Q4)
    for bad in [(0, 1, 64, 1), (1, 0, 64, 1), (1, 1, 96, 1), (1, 1, 64, 0), (1, 1, 64, (1 << 30) + 1), (300, 300, 64, 1),
                (1 << 40, 1 << 40, 64, 1)]:
        assert size(*bad) == 0
    assert work(1, 1, 8, 4, 256, 32768, 0) > 0
    assert work(1, 1, 4, 1, 256, 32, 0) == 0
    for bad in [(0, 1, 8, 4, 256, 100, 0), (1, 0, 8, 4, 256, 100, 0), (1, 101, 8, 4, 256, 100, 0), (1, 1, 6, 4, 256, 100, 0),
                (1, 1, 68, 4, 256, 100, 0), (1, 1, 8, 4, 96, 100, 0), (1, 1, 8, 4, 256, 100, -1), (1, 1 << 20, 8, 4, 256, 1 << 30, 0)]:
        assert work(*bad) == 0


def _store(**change):
    v = dict(q=A, k=A, v=A, positions=A, seqs=0, q_weight=A, k_weight=A, inv_freq=A, q_out=A, k_cache=A, v_cache=A,
             q_stride=1024, k_stride=512, v_stride=512, T=3, H=8, G=4, d=128, B=2, L=100, weight_offset=1.0, eps=1e-6,
             in_dtype=1, format=1)
    v.update(change)
    return LIB.q4nx_kv_store(q4._KV_STORE_ARGS.pack(*v.values()), None)


def test_store_refusals():
    assert LIB.q4nx_kv_store(None, None) == q4.Q4NX_ERR_INVALID_ARG
    for name in ("q", "k", "v", "positions", "q_out", "k_cache", "v_cache"):
        assert _store(**{name: 0}) == q4.Q4NX_ERR_INVALID_ARG, name
    for change in (dict(in_dtype=2), dict(in_dtype=-1), dict(format=7), dict(weight_offset=float("nan")),
                   dict(eps=float("inf")), dict(eps=-1e-6)):
        assert _store(**change) == q4.Q4NX_ERR_INVALID_ARG, change
    for change in (dict(T=0), dict(T=(1 << 24) + 1), dict(H=0), dict(H=65536), dict(G=0), dict(B=0), dict(d=96), dict(L=0),
                   dict(L=(1 << 30) + 1), dict(B=40000, G=2), dict(q_stride=1016), dict(k_stride=504), dict(v_stride=-512),
                   dict(v_stride=(1 << 32) + 8)):
        assert _store(**change) == q4.Q4NX_ERR_SHAPE, change
    for name in ("q", "k", "v", "q_weight", "k_weight", "inv_freq", "q_out", "k_cache", "v_cache"):
        assert _store(**{name: A + 8}) == q4.Q4NX_ERR_ALIGNMENT, name
    for change in (dict(positions=A + 2), dict(seqs=A + 2), dict(q_stride=1028), dict(in_dtype=0, k_stride=514)):
        assert _store(**change) == q4.Q4NX_ERR_ALIGNMENT, change
    # In place for float32 and for rows with gaps: a wave would write what another has yet to read.
    for change in (dict(in_dtype=0), dict(q_stride=1032), dict(T=1, q_stride=2048)):
        assert _store(**change) == q4.Q4NX_ERR_INVALID_ARG, change
    assert "q4nx_kv_store" in LIB.q4nx_last_error().decode()


def _load(k=A, v=A, positions=A, seqs=0, T=3, G=4, d=128, B=2, L=100, ko=A, vo=A, dtype=0):
    return LIB.q4nx_kv4_load(k, v, positions, seqs, T, G, d, B, L, ko, vo, dtype, None)


def test_load_refusals():
    for name in ("k", "v", "positions", "ko", "vo"):
        assert _load(**{name: 0}) == q4.Q4NX_ERR_INVALID_ARG, name
    assert _load(dtype=3) == q4.Q4NX_ERR_INVALID_ARG
    for change in (dict(T=0), dict(G=0), dict(d=32), dict(B=0), dict(L=0), dict(B=2, G=40000), dict(B=1, T=1 << 24, G=65535),
                   dict(T=(1 << 24), G=9), dict(T=(1 << 23), G=9, d=256)):
        assert _load(**change) == q4.Q4NX_ERR_SHAPE, change
    for change in (dict(k=A + 4), dict(v=A + 8), dict(ko=A + 2), dict(vo=A + 4), dict(positions=A + 1), dict(seqs=A + 2)):
        assert _load(**change) == q4.Q4NX_ERR_ALIGNMENT, change


def _attend(q=A, k=A, v=A, lens=A, B=1, T=1, H=8, G=4, d=256, L=32768, window=0, scale=0.0625, o=A, dtype=0, work=A,
            nbytes=1 << 40):
    return LIB.q4nx_kv4_attention(q, k, v, lens, B, T, H, G, d, L, window, scale, o, dtype, work, nbytes, None)


def test_attention_refusals():
    for change in (dict(q=0), dict(k=0), dict(v=0), dict(lens=0), dict(o=0), dict(dtype=2), dict(scale=float("inf")),
                   dict(scale=float("nan")), dict(work=0)):
        assert _attend(**change) == q4.Q4NX_ERR_INVALID_ARG, change
    for change in (dict(B=0), dict(T=0), dict(T=32769), dict(H=6), dict(H=68), dict(G=0), dict(d=512), dict(L=0),
                   dict(window=-1), dict(window=(1 << 30) + 1), dict(B=20000), dict(T=1 << 20, L=1 << 30),
                   dict(B=60000, H=1, G=1, T=20000), dict(B=16384, T=8193, H=8, G=1)):
        assert _attend(**change) == q4.Q4NX_ERR_SHAPE, change
    for change in (dict(q=A + 8), dict(k=A + 4), dict(v=A + 4), dict(o=A + 8), dict(work=A + 8), dict(lens=A + 2)):
        assert _attend(**change) == q4.Q4NX_ERR_ALIGNMENT, change
    need = LIB.q4nx_kv4_workspace_size(1, 1, 8, 4, 256, 32768, 0)
    assert _attend(nbytes=need - 1) == q4.Q4NX_ERR_BUFFER_TOO_SMALL


def test_binding_checks_sizes_and_types():
    torch = pytest.importorskip("torch")
    t = torch.zeros(4096, dtype=torch.bfloat16)
    with pytest.raises(ValueError):        # not a GPU tensor
        q4.q4nx_kv_store(t, t, t, t, t, t, t, 1, 8, 4, 128, 1, 32)
    with pytest.raises(ValueError):        # caches too small
        q4.q4nx_kv4_attention(t, t, t, t, 1, 1, 8, 4, 128, 32768, 0, 1.0, t)
    with pytest.raises(ValueError):
        q4.q4nx_kv4_load(t, t, t, t, t, 1, 4, 128, 1, 32768)


def test_refusals_under_the_host_sanitizers():
    from test_host_sanitizer import ROOT, _build_module, _stale
    import os
    import subprocess
    import sys
    b = _build_module()
    if os.environ.get("Q4NX_LIBRARY") or not os.path.exists(b.hipcc()):
        pytest.skip("the child itself, or no hipcc")
    if _stale(b.ASAN_LIB):
        b.build(sanitize=True)
    env = dict(os.environ, Q4NX_LIBRARY=b.ASAN_LIB, LD_PRELOAD=b.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and " passed" in out and "runtime error" not in out, out[-4000:]


def test_struct_is_the_headers():
    assert q4._KV_STORE_ARGS.size == 11 * ctypes.sizeof(ctypes.c_void_p) + 9 * 8 + 4 * 4
