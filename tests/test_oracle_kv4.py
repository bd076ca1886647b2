"""Pins of the 4-bit KV cache oracle: facts that it does not define itself."""
import numpy as np
import pytest

import oracle
from oracle import kv4
from oracle.attention import decode_attention


@pytest.mark.parametrize("address", [kv4.k_address, kv4.v_address])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_value_has_a_nibble_of_its_own(address, d):
    P = 64
    p, i = np.meshgrid(np.arange(P), np.arange(d), indexing="ij")
    byte, nibble, pair = address(p, i, P, d)
    assert sorted((2 * byte + nibble).ravel()) == list(range(P * d))
    groups = {}
    for key, at in zip(zip(p.ravel(), (i // 32).ravel()), pair.ravel()):
        groups.setdefault(key, set()).add(int(at))
    assert all(len(v) == 1 for v in groups.values())
    assert sorted(v.pop() for v in groups.values()) == list(range(P * d // 32))


def test_addresses_by_hand():
    # K at d = 64: position 3, value 13 = word 1, byte 1, high nibble; group 0 of 2
    assert kv4.k_address(3, 13, 32, 64) == (3 * 32 + 4 + 1, 1, 6)
    # V at d = 128: position 32 + 16 + 4*2 + 3, value 64 + 32 + 16 + 5
    assert kv4.v_address(59, 117, 64, 128) == (2048 + 1024 + ((2 * 16 + 5) * 2 + 1) * 8 + 4 + 3, 1, 128 + 96 + 16 + 4 + 3)


def test_rows_come_back_as_the_quantizer_left_them():
    rng = np.random.default_rng(1)
    d, L, heads = 128, 40, 3
    rows = rng.standard_normal((5, d)).astype(np.float32)
    codes, s, o = oracle.quantize(rows)
    want = oracle.dequant_bf16(codes, s, o)
    for address in (kv4.k_address, kv4.v_address):
        cache = rng.integers(0, 256, heads * 64 * d * 5 // 8).astype(np.uint8)
        kv4.write_rows(cache, rows, [0, 2, 1, 2, 0], [0, 39, 17, 38, 1], heads, L, address)
        got = kv4.read_rows(cache, [0, 2, 1, 2, 0], [0, 39, 17, 38, 1], heads, L, d, address)
        assert np.array_equal(got, want)


def test_norm_and_rotation_special_cases():
    x = np.zeros((2, 1, 64), np.float32)
    x[:, 0, 3], x[:, 0, 35] = 3.0, 4.0
    one = np.full(64, 0x3F80, np.uint16)
    y = kv4.normed_rotated(x, one, 0.0, 0.0, [0, 0], None)
    assert np.allclose(np.square(y).mean(-1), 1.0) and np.allclose(y[0, 0, 3] / y[0, 0, 35], 0.75)
    f = np.zeros(32, np.float32)
    f[3] = np.float32(np.pi / 2)
    z = kv4.normed_rotated(x, None, 0.0, 0.0, [0, 1], f)
    assert np.array_equal(z[0], x[0].astype(np.float64))                 # position 0: as it was
    assert np.allclose(z[1, 0, [3, 35]], [-4.0, 3.0], atol=1e-6)         # a quarter turn


def test_attention_reduces_to_the_single_token_oracle():
    rng = np.random.default_rng(2)
    bits = lambda *s: oracle.f32_to_bf16(rng.standard_normal(s, dtype=np.float32))  # noqa: E731
    q, K, V = bits(3, 4, 64), bits(2, 20, 64), bits(2, 20, 64)
    for window in (0, 1, 5):
        o = kv4.attention(q, K, V, 20, window, 0.125)[0]
        for t in range(3):
            assert np.allclose(o[t], decode_attention(q[t], K, V, 17 + t, window, 0.125)[0], rtol=1e-12)
    assert not kv4.attention(q, K, V, 2, 0, 0.125)[0][0].any()            # row 0 stands before the start
