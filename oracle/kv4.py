"""The 4-bit K/V cache, reference (test infrastructure only).

A row's 32 consecutive elements share a power p and count 2^(p - 127) each;
an element's code is a sign (bit 3) and one of eight sizes. For bf16 inputs:

  * p is the least value from 1 to 252 with max |x| <= 7 * 2^(p - 127) (252 if
    there is none);
  * the code is the size nearest to |x| / 2^(p - 127), of two equally near the
    one with the even code, with x's sign;
  * a group that holds an infinity or a NaN has p = 255 and codes 0, and all of
    its elements read as NaN.

Written element by element, in exact fractions where a choice depends on it.
"""

from __future__ import annotations

from fractions import Fraction

import numpy as np

from .attention import decode_bf16

SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ST_GAMMA = 1
ST_KVLEN = 2


def power_of(top: float) -> int:
    """The power of a group whose largest magnitude is `top` (finite)."""
    for p in range(1, 253):
        if Fraction(top) <= 7 * Fraction(2) ** (p - 127):
            return p
    return 252


def code_of(x: float, p: int) -> int:
    r = abs(Fraction(x)) / Fraction(2) ** (p - 127)
    near = min(abs(r - Fraction(s)) for s in SIZES)
    best = [c for c, s in enumerate(SIZES) if abs(r - Fraction(s)) == near]
    code = best[0] if len(best) == 1 else next(c for c in best if c % 2 == 0)
    return code | (8 if np.signbit(x) else 0)


_POWERS: dict = {}
_CODES: dict = {}


def round_group(bits):
    """bf16 bits [32] -> (codes [32], p)."""
    bits = np.asarray(bits, np.uint16)
    mags = bits & 0x7FFF
    top = int(mags.max())
    if top >= 0x7F80:
        return np.zeros(32, np.uint8), 255
    if top not in _POWERS:
        _POWERS[top] = power_of(float(decode_bf16(np.uint16(top))))
    p = _POWERS[top]
    codes = np.empty(32, np.uint8)
    for n, b in enumerate(bits.tolist()):
        if (b, p) not in _CODES:
            _CODES[b, p] = code_of(float(decode_bf16(np.uint16(b))), p)
        codes[n] = _CODES[b, p]
    return codes, p


def to_4_bits(bits):
    """bf16 bits [..., D] -> (codes u8 [..., D/2], powers u8 [..., D/32])."""
    bits = np.asarray(bits, np.uint16)
    flat = bits.reshape(-1, 32)
    codes = np.empty(flat.shape, np.uint8)
    powers = np.empty(flat.shape[0], np.uint8)
    for r in range(flat.shape[0]):
        codes[r], powers[r] = round_group(flat[r])
    codes = codes.reshape(bits.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), powers.reshape(bits.shape[:-1] + (-1,))


def values(codes, powers):
    """What codes and powers stand for, fp64 [..., D]."""
    codes = np.asarray(codes, np.uint8)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.asarray(SIZES)[c & 7] * np.where(c & 8, -1.0, 1.0)
    p = np.asarray(powers).astype(np.int64)
    unit = np.where(p == 255, np.nan, np.exp2(np.where(p == 255, 0, p - 127).astype(np.float64)))
    return v * np.repeat(unit, 32, axis=-1)


def append(cache, mask, kv_len, k_new, v_new, gamma, phys_len=None):
    """cache = (k_codes, k_powers, v_codes, v_powers). Returns (cache, mask, kv_len,
    (k_seen, v_seen) fp64, wrote [B, gmax+1], status) as new arrays; rows that are not
    written have wrote False and NaN in the seen values."""
    kc, kp, vc, vp = (np.array(t, copy=True) for t in cache)
    m = None if mask is None else np.array(mask, copy=True)
    kl = np.array(kv_len, dtype=np.int64, copy=True)
    B, Hkv, L_cap, _ = kc.shape
    G1 = k_new.shape[1]
    seen = [np.full(k_new.shape, np.nan) for _ in range(2)]
    wrote = np.zeros((B, G1), dtype=bool)
    status = 0
    for b in range(B):
        g = int(gamma[b])
        if not 0 <= g < G1:
            status |= ST_GAMMA
            continue
        cur = int(kl[b]) if phys_len is None else int(phys_len)
        if not 0 <= kl[b] <= L_cap or cur < 0 or cur + g + 1 > L_cap:
            status |= ST_KVLEN
            continue
        n = g + 1
        for new, codes, powers, s in ((k_new, kc, kp, seen[0]), (v_new, vc, vp, seen[1])):
            c4, p4 = to_4_bits(new[b, :n])  # [n, Hkv, .]
            codes[b, :, cur:cur + n] = c4.swapaxes(0, 1)
            powers[b, :, cur:cur + n] = p4.swapaxes(0, 1)
            s[b, :n] = values(c4, p4)
        if m is not None:
            m[b, cur:cur + n] = 1
        kl[b] = cur + n
        wrote[b, :n] = True
    return (kc, kp, vc, vp), m, kl.astype(np.int32), seen, wrote, status
