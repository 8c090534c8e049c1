"""Host-side argument checks of the calls around the attention, on the CPU: every
bad argument is refused before anything touches the device."""

import ctypes
import os

import pytest
import torch

from paper_2505_07680_amd import _lib

no_device = pytest.mark.skipif(
    torch.cuda.device_count() > 0, reason="host-only argument checks"
)
EINVAL, EUNSUPPORTED, EWORKSPACE, ELAUNCH = _lib.SR_EINVAL, _lib.SR_EUNSUPPORTED, _lib.SR_EWORKSPACE, _lib.SR_ELAUNCH


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2505_07680_amd.build import build

        build()
    return _lib.load()


P = ctypes.c_void_p(4096)  # never dereferenced: every case ends before a launch
ODD = ctypes.c_void_p(4104)


def _refusals(call, good, cases):
    assert call(*good) == ELAUNCH  # fine but for the device, of which there is none here
    for at, value, want in cases:
        args = list(good)
        args[at] = value
        assert call(*args) == want, (at, value)


def test_position_bit_has_a_text(lib):
    assert b"position" in lib.specrouter_status_string(_lib.SR_ST_POSITION)


@no_device
def test_norm_rope(lib):
    # q, stride, k, stride, wq, wk, dtype, eps, table, max_pos, rot, pairs, pos, gamma, qo, ko, B, gmax, Hq, Hkv, D, status, stream
    good = [P, 512, P, 128, None, None, 0, 1e-6, P, 100, 64, 0, P, P, ctypes.c_void_p(8192), ctypes.c_void_p(16384),
            2, 3, 8, 2, 64, None, None]
    cases = [(i, None, EINVAL) for i in (0, 2, 8, 12, 13, 14, 15)]
    cases += [(i, ODD, EINVAL) for i in (0, 2, 4, 5, 8, 14, 15)]
    cases += [(1, 504, EINVAL), (1, 516, EINVAL), (3, 120, EINVAL), (6, 2, EUNSUPPORTED), (7, -1e-6, EINVAL),
              (7, float("nan"), EINVAL), (7, float("inf"), EINVAL), (9, 0, EINVAL), (10, 0, EINVAL), (10, 24, EINVAL),
              (10, 80, EINVAL), (16, 0, EINVAL), (17, -1, EINVAL), (18, 0, EINVAL), (19, 0, EINVAL),
              (18, 1 << 20, EINVAL), (20, 96, EUNSUPPORTED), (17, 2 ** 31 - 1, EINVAL), (16, 2 ** 31 - 1, EINVAL)]
    _refusals(lib.specrouter_qk_norm_rope, good, cases)
    apart = list(good)
    apart[1], apart[14] = 1024, P  # in place, with the rows of a wider projection
    assert lib.specrouter_qk_norm_rope(*apart) == EINVAL
    apart[1] = 512
    assert lib.specrouter_qk_norm_rope(*apart) == ELAUNCH


@no_device
def test_kv4_append(lib):
    # k, stride, v, stride, gamma, kc, kp, vc, vp, mask, kv_len, shared, k_seen, v_seen, B, gmax, Hkv, D, L_cap, status, stream
    good = [P, 128, P, 128, P, P, P, P, P, None, P, None, None, None, 2, 3, 2, 64, 100, None, None]
    cases = [(i, None, EINVAL) for i in (0, 2, 4, 5, 6, 7, 8, 10)]
    cases += [(i, ODD, EINVAL) for i in (0, 2, 5, 7, 12, 13)]
    cases += [(i, ctypes.c_void_p(4098), EINVAL) for i in (6, 8)]
    cases += [(1, 120, EINVAL), (3, 132, EINVAL), (14, 0, EINVAL), (14, 65536, EINVAL), (15, -1, EINVAL),
              (15, 100, EINVAL), (16, 0, EINVAL), (17, 32, EUNSUPPORTED), (18, 0, EINVAL), (18, (1 << 22) + 1, EINVAL)]
    _refusals(lib.specrouter_kv4_append, good, cases)


@no_device
def test_window_attention(lib):
    # q, k, v, mask, kv_len, gamma, out, dtype, B, gmax, Hq, Hkv, D, L_cap, window, sinks, scale, ws, bytes, status, stream
    good = [P, P, P, None, P, P, P, 1, 2, 4, 8, 2, 128, 512, 64, 4, 0.1, None, 0, None, None]
    cases = [(i, None, EINVAL) for i in (0, 1, 2, 4, 5, 6)] + [(i, ODD, EINVAL) for i in (0, 1, 2, 6)]
    cases += [(7, 2, EUNSUPPORTED), (8, 0, EINVAL), (9, 17, EINVAL), (9, -1, EINVAL), (11, 3, EINVAL),
              (12, 96, EUNSUPPORTED), (13, 4, EINVAL), (13, (1 << 22) + 1, EINVAL), (14, 0, EINVAL), (14, -5, EINVAL),
              (15, -1, EINVAL)]
    cases += [(16, s, EINVAL) for s in (0.0, -0.1, float("nan"), float("inf"))]
    _refusals(lib.specrouter_verify_attention_window, good, cases)
    assert lib.specrouter_verify_attention_window_workspace_size(2, 4, 8, 2, 128, 512, 0, 4) == 0


@no_device
def test_kv4_attention(lib):
    # q, kc, kp, vc, vp, mask, kv_len, gamma, out, dtype, B, gmax, Hq, Hkv, D, L_cap, window, sinks, scale, ws, bytes, ...
    good = [P, P, P, P, P, None, P, P, P, 0, 2, 4, 8, 2, 64, 512, 0, 0, 0.1, None, 0, None, None]
    cases = [(i, None, EINVAL) for i in (0, 1, 2, 3, 4, 6, 7, 8)] + [(i, ODD, EINVAL) for i in (0, 1, 3, 8)]
    cases += [(i, ctypes.c_void_p(4098), EINVAL) for i in (2, 4)]
    cases += [(9, 5, EUNSUPPORTED), (10, 65536, EINVAL), (11, 17, EINVAL), (12, 9, EINVAL), (14, 32, EUNSUPPORTED),
              (15, 4, EINVAL), (16, -1, EINVAL), (17, -1, EINVAL)]
    cases += [(18, s, EINVAL) for s in (0.0, float("nan"), float("inf"))]
    _refusals(lib.specrouter_verify_attention_kv4, good, cases)
    assert lib.specrouter_verify_attention_kv4_workspace_size(2, 4, 8, 3, 64, 512, 0, 0) == 0


@no_device
def test_rows_that_would_overwrite_each_other(lib):
    """Outputs that are another argument, in place with wider rows, and a cursor among the lengths."""
    Q, K = ctypes.c_void_p(8192), ctypes.c_void_p(16384)
    good = [P, 512, Q, 128, None, None, 0, 1e-6, P, 100, 64, 0, P, P, P, Q, 2, 3, 8, 2, 64, None, None]
    _refusals(lib.specrouter_qk_norm_rope, good, [(14, Q, EINVAL), (15, P, EINVAL), (15, K, ELAUNCH)])
    lens = ctypes.c_void_p(65536)
    good = [P, 128, Q, 128, P, P, P, P, P, None, lens, None, P, Q, 2, 3, 2, 64, 100, None, None]
    cases = [(1, 256, EINVAL), (3, 256, EINVAL), (12, Q, EINVAL), (13, P, EINVAL), (11, lens, EINVAL),
             (11, ctypes.c_void_p(65540), EINVAL), (11, ctypes.c_void_p(65544), ELAUNCH)]
    _refusals(lib.specrouter_kv4_append, good, cases)
    same = list(good)
    same[12] = same[13] = K
    assert lib.specrouter_kv4_append(*same) == EINVAL


@no_device
def test_more_threads_than_a_launch_counts(lib):
    # 2^26 tokens of one query and one key head are 2^26 waves, 2^32 threads
    good = [P, 64, P, 64, None, None, 0, 1e-6, P, 100, 64, 0, P, P, ctypes.c_void_p(8192), ctypes.c_void_p(16384),
            1, (1 << 26) - 5, 1, 1, 64, None, None]
    _refusals(lib.specrouter_qk_norm_rope, good, [(17, (1 << 26) - 1, EINVAL)])


class _Shape:
    """A tensor's outside: what a call checks before it takes any address."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0):
        self.shape, self.dtype, self.device = shape, dtype, device

    get_device = lambda self: self.device
    is_contiguous = lambda self: True
    dim = lambda self: len(self.shape)
    numel = lambda self: int(__import__("math").prod(self.shape))

    def data_ptr(self):
        raise AssertionError("the call went through")

    def stride(self):
        raise AssertionError("the call went through")


I32, U8 = torch.int32, torch.uint8


@pytest.fixture
def device_0(monkeypatch):
    monkeypatch.setattr(_lib, "_current", lambda: 0)


def _rope_call(**change):
    a = dict(q=_Shape(2, 3, 8, 64), k=_Shape(2, 3, 2, 64), q_weight=None, k_weight=None, eps=1e-6,
             rope_table=_Shape(100, 64, dtype=torch.float32), position=_Shape(2, dtype=I32), gamma=_Shape(2, dtype=I32),
             q_out=_Shape(2, 3, 8, 64), k_out=_Shape(2, 3, 2, 64))
    _lib.specrouter_qk_norm_rope(**{**a, **change})


def _append_call(**change):
    codes, powers = _Shape(2, 2, 100, 32, dtype=U8), _Shape(2, 2, 100, 2, dtype=U8)
    a = dict(k_new=_Shape(2, 3, 2, 64), v_new=_Shape(2, 3, 2, 64), gamma=_Shape(2, dtype=I32), k_codes=codes,
             k_powers=powers, v_codes=codes, v_powers=powers, cache_mask=None, kv_len=_Shape(2, dtype=I32))
    _lib.specrouter_kv4_append(**{**a, **change})


def _window_call(**change):
    a = dict(q=_Shape(2, 3, 8, 64), k_cache=_Shape(2, 2, 100, 64), v_cache=_Shape(2, 2, 100, 64), cache_mask=None,
             kv_len=_Shape(2, dtype=I32), gamma=_Shape(2, dtype=I32), out=_Shape(2, 3, 8, 64), scale=0.125, window=16)
    _lib.specrouter_verify_attention_window(**{**a, **change})


def _kv4_call(**change):
    codes, powers = _Shape(2, 2, 100, 32, dtype=U8), _Shape(2, 2, 100, 2, dtype=U8)
    a = dict(q=_Shape(2, 3, 8, 64), k_codes=codes, k_powers=powers, v_codes=codes, v_powers=powers, cache_mask=None,
             kv_len=_Shape(2, dtype=I32), gamma=_Shape(2, dtype=I32), out=_Shape(2, 3, 8, 64), scale=0.125)
    _lib.specrouter_verify_attention_kv4(**{**a, **change})


WRONG_STATUS = (dict(status=_Shape(1, dtype=torch.int64)), dict(status=_Shape(1, dtype=I32, device=1)))


@pytest.mark.parametrize("call, changes", [
    (_rope_call, [dict(k_weight=_Shape(64, dtype=torch.float64)), dict(q_weight=_Shape(64, dtype=torch.float64)),
                  dict(q_weight=_Shape(64), k_weight=_Shape(64, dtype=torch.float32)),
                  dict(k=_Shape(2, 3, 64)), dict(k=_Shape(2, 4, 2, 64)), dict(k_out=_Shape(2, 3, 8, 64)),
                  dict(position=_Shape(2, 1, dtype=I32)), dict(gamma=_Shape(3, dtype=I32)),
                  dict(rope_table=_Shape(1 << 31, 64, dtype=torch.float32))]),
    (_append_call, [dict(k_codes=_Shape(2, 100, 32, dtype=U8)), dict(v_codes=_Shape(2, 2, 99, 32, dtype=U8)),
                    dict(k_powers=_Shape(2, 2, 100, 1, dtype=U8)), dict(kv_len=_Shape(2, dtype=torch.int64)),
                    dict(k_seen=_Shape(2, 3, 2, 128)), dict(shared_len=_Shape(2, dtype=I32))]),
    (_window_call, [dict(window=2 ** 32 + 5), dict(window=-2 ** 32 + 5), dict(sinks=2 ** 32), dict(k_cache=_Shape(2, 2, 64)),
                    dict(v_cache=_Shape(2, 2, 99, 64)), dict(out=_Shape(2, 3, 8, 64, dtype=torch.float16)),
                    dict(kv_len=_Shape(1, dtype=I32))]),
    (_kv4_call, [dict(window=2 ** 32 + 5), dict(sinks=2 ** 32), dict(k_codes=_Shape(2, 100, 32, dtype=U8)),
                 dict(v_powers=_Shape(2, 2, 100, 1, dtype=U8)), dict(q=_Shape(2, 3, 8, 64, dtype=torch.float16)),
                 dict(cache_mask=_Shape(2, 99, dtype=U8))]),
])
def test_bindings_refuse_before_they_take_an_address(lib, device_0, call, changes):
    with pytest.raises(AssertionError, match="went through"):
        call()
    for change in (*changes, *WRONG_STATUS):
        with pytest.raises((ValueError, TypeError)):
            call(**change)
