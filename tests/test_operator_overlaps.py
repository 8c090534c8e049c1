"""Outputs that start inside another argument of specrouter_qk_norm_rope and
specrouter_kv4_append: the binding refuses them (on the CPU, with the library's calls counted)."""

import pytest
import torch

from paper_2505_07680_amd import _lib

B, ROWS, HQ, HKV, D, CAP = 2, 3, 4, 2, 64, 10
NQ, NK = B * ROWS * HQ * D, B * ROWS * HKV * D


@pytest.fixture
def calls(monkeypatch):
    """The names of the library calls that were made, on CPU tensors."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(_lib, "_current", lambda: -1)
    monkeypatch.setattr(_lib, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0)
    return made


class Memory:
    """One allocation; take(at, *shape): a contiguous view from element `at` on."""

    def __init__(self, n, dtype=torch.bfloat16):
        self.flat = torch.zeros(n, dtype=dtype)

    def take(self, at, *shape):
        n = 1
        for s in shape:
            n *= s
        return self.flat[at:at + n].view(*shape)


def _rope(q, k, q_out, k_out):
    i = torch.zeros(B, dtype=torch.int32)
    _lib.specrouter_qk_norm_rope(q, k, None, None, 1e-6, torch.zeros(8, D), i, i, q_out, k_out)


def _heads(m, at, H):
    return m.take(at, B, ROWS, H, D)


@pytest.mark.parametrize("name, q, k, q_out, k_out", [
    ("q_out inside q", 0, 20000, 8, 30000),
    ("q_out ends inside q", 8, 20000, 0, 30000),
    ("q_out inside k", 0, 20000, 20000 + NK - 8, 30000),
    ("q_out ends inside k", 0, 20000, 20000 - NQ + 8, 30000),
    ("q_out at k", 0, 20000, 20000, 30000),
    ("k_out inside q", 0, 20000, 10000, NQ - 8),
    ("k_out ends inside k", 0, 20000, 10000, 20000 - 8),
    ("k_out inside q_out", 0, 20000, 10000, 10000 + NQ - 8),
    ("k_out at q_out", 0, 20000, 10000, 10000),
    ("in place, k inside q", 0, HQ * D, 0, 30000),
])
def test_norm_rope_refuses(calls, name, q, k, q_out, k_out):
    m = Memory(40000)
    with pytest.raises(ValueError, match="must not overlap"):
        _rope(_heads(m, q, HQ), _heads(m, k, HKV), _heads(m, q_out, HQ), _heads(m, k_out, HKV))
    assert calls == []


@pytest.mark.parametrize("name, q, k, q_out, k_out", [
    ("one after the other", 0, NQ, NQ + NK, 2 * NQ + NK),
    ("the outputs first", NQ + NK, 2 * NQ + NK, 0, NQ),
    ("in place", 0, NQ, 0, NQ),
    ("queries in place", 0, NQ, 0, 30000),
    ("keys of the queries' rows", 0, 0, 0, 30000),
    ("queries of the keys' rows", 0, 0, 30000, 0),
])
def test_norm_rope_takes(calls, name, q, k, q_out, k_out):
    m = Memory(40000)
    _rope(_heads(m, q, HQ), _heads(m, k, HKV), _heads(m, q_out, HQ), _heads(m, k_out, HKV))
    assert calls == ["specrouter_qk_norm_rope"]


def test_norm_rope_views_of_one_projection(calls):
    """Outputs between the rows of a projection touch none of them; at its rows' ends they do."""
    wide = HQ * D * B * ROWS * 4
    m = Memory(wide * B * ROWS + 64)
    x = m.take(0, B, ROWS, wide)
    q, k = x[..., :HQ * D].unflatten(-1, (HQ, D)), x[..., HQ * D:(HQ + HKV) * D].unflatten(-1, (HKV, D))
    between = (HQ + HKV) * D
    _rope(q, k, _heads(m, between, HQ), _heads(m, between + NQ, HKV))
    _rope(q, k, _heads(m, wide - NQ, HQ), _heads(m, wide + between, HKV))
    assert len(calls) == 2
    for q_out, k_out in ((between - 8, between + NQ), (wide - NQ + 8, between), (between, wide - NK + 8),
                         (between, between + NQ - 8)):
        with pytest.raises(ValueError, match="must not overlap"):
            _rope(q, k, _heads(m, q_out, HQ), _heads(m, k_out, HKV))
    assert len(calls) == 2


def _append(k_new, v_new, cache, k_seen, v_seen):
    i = torch.zeros(B, dtype=torch.int32)
    _lib.specrouter_kv4_append(k_new, v_new, i, *cache, None, i, k_seen=k_seen, v_seen=v_seen)


CODES, POWERS = B * HKV * CAP * D // 2, B * HKV * CAP * D // 32


def _cache(flat, at):
    """The four arrays one after the other from byte `at` of a byte tensor on."""
    out = []
    for n in (D // 2, D // 32, D // 2, D // 32):
        size = B * HKV * CAP * n
        out.append(flat[at:at + size].view(B, HKV, CAP, n))
        at += size
    return out


@pytest.mark.parametrize("name, k, v, k_seen, v_seen", [
    ("k_seen inside k_new", 0, 5000, 8, None),
    ("k_seen ends inside v_new", 0, 5000, 5000 - NK + 8, None),
    ("v_seen inside k_new", 0, 5000, None, NK - 8),
    ("v_seen inside v_new", 0, 5000, 0, 5008),
    ("v_seen inside k_seen", 0, 5000, 10000, 10000 + NK - 8),
    ("k_seen in the first codes", 0, 5000, 20000, None),
    ("v_seen ends in the first codes", 0, 5000, None, 20000 - NK + 8),
    ("k_seen from K's last powers on", 0, 5000, 20000 + (CODES + POWERS) // 2 - 8, None),
    ("v_seen from V's last powers on", 0, 5000, 0, 20000 + (CODES + POWERS) - 8),
])
def test_kv4_append_refuses(calls, name, k, v, k_seen, v_seen):
    m = Memory(40000)
    at = lambda e: None if e is None else _heads(m, e, HKV)
    with pytest.raises(ValueError, match="must not overlap"):
        _append(at(k), at(v), _cache(m.flat.view(torch.uint8), 40000), at(k_seen), at(v_seen))
    assert calls == []


@pytest.mark.parametrize("name, k, v, k_seen, v_seen", [
    ("in place", 0, NK, 0, NK),
    ("one of them", 0, NK, None, NK),
    ("around the cache", 0, NK, 20000 - NK, 20000 + CODES + POWERS),
    ("apart", 0, NK, 2 * NK, 3 * NK),
    ("none", 0, NK, None, None),
])
def test_kv4_append_takes(calls, name, k, v, k_seen, v_seen):
    m = Memory(40000)
    at = lambda e: None if e is None else _heads(m, e, HKV)
    _append(at(k), at(v), _cache(m.flat.view(torch.uint8), 40000), at(k_seen), at(v_seen))
    assert calls == ["specrouter_kv4_append"]
