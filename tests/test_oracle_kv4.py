"""Pins of the 4-bit cache's reference: the definition's own properties over every bf16 value."""

import numpy as np

from oracle import kv4
from oracle.attention import decode_bf16


def _group(values):
    x = np.zeros(32, np.float32)
    x[: len(values)] = values
    return (x.view(np.uint32) >> 16).astype(np.uint16)


def test_ties_go_to_the_even_code_and_signs_stay():
    # with a largest element of 7 the power is 1
    x = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5, 0.375, 6.5, -0.0]
    codes, p = kv4.round_group(_group(x))
    assert p == 127
    assert codes[: len(x)].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14, 1, 7, 8]


def test_power_is_the_least_that_keeps_the_largest_below_seven():
    for bits in list(range(0, 0x7F80, 13)) + [0x7F7F]:
        p = kv4.round_group(np.full(32, bits, np.uint16))[1]
        top = float(decode_bf16(np.uint16(bits)))
        assert 1 <= p <= 252
        assert p == 252 or top <= 7.0 * 2.0 ** (p - 127)
        assert p == 1 or top > 7.0 * 2.0 ** (p - 128)
        # the exponent, one more above a mantissa of 1.75, less 2
        assert p == min(max(((bits + 0x1F) >> 7) - 2, 1), 252)


def test_error_is_at_most_half_a_step_of_the_largest():
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(50, 32)) * np.exp(rng.normal(size=(50, 1)) * 5)).astype(np.float32)
    bits = (x.view(np.uint32) >> 16).astype(np.uint16)
    v = decode_bf16(bits)
    codes, powers = kv4.to_4_bits(bits)
    got = kv4.values(codes, powers)
    assert (np.abs(got - v) <= 2.0 ** (powers.astype(float) - 127)).all()
    # and rounding again changes nothing where no element sat above 6
    again = (got.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    c2, p2 = kv4.to_4_bits(again)
    np.testing.assert_array_equal(kv4.values(c2, p2), got)


def test_infinite_and_nan_groups_read_as_nan():
    for bad in (0x7F80, 0xFF80, 0x7FC1):
        g = _group([1, 2, 3])
        g[5] = bad
        codes, p = kv4.round_group(g)
        assert p == 255 and not codes.any()
        row = np.concatenate([g, _group([1.0])])
        v = kv4.values(*kv4.to_4_bits(row))
        assert np.isnan(v[:32]).all() and v[32] == 1.0


def test_append_places_rows_and_flags_bad_sequences():
    rng = np.random.default_rng(4)
    B, Hkv, L, D, G1 = 5, 2, 12, 64, 3
    new = (rng.normal(size=(B, G1, Hkv, D)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    cache = tuple(np.full((B, Hkv, L, w), 7, np.uint8) for w in (D // 2, D // 32, D // 2, D // 32))
    mask = np.zeros((B, L), np.uint8)
    out, m, kl, seen, wrote, st = kv4.append(cache, mask, [0, 9, 11, 13, 4], new, new[:, :, ::-1], [2, 2, 1, 0, 3])
    assert st == kv4.ST_GAMMA | kv4.ST_KVLEN
    assert kl.tolist() == [3, 12, 11, 13, 4]
    assert m.sum(1).tolist() == [3, 3, 0, 0, 0] and wrote.sum(1).tolist() == [3, 3, 0, 0, 0]
    np.testing.assert_array_equal(kv4.values(out[0], out[1])[1, 1, 9:], seen[0][1, :, 1])
    np.testing.assert_array_equal(kv4.values(out[2], out[3])[0, 0, :3], seen[1][0, :, 0])
    assert (out[0][0, :, 3:] == 7).all() and (out[0][2] == 7).all()
