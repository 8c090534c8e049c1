"""Norm and rotation, append and attention where byte offsets pass 31 and 32 bits:
the longest caches, many of them, and tensors of more than 2^31 elements. The
results are those of small tensors that hold the same rows."""

import numpy as np
import pytest
import torch

from operator_util import Inputs, bf16, check, normal_bits, say

pytestmark = pytest.mark.gpu
CAP = 1 << 22  # the longest cache
BF = dict(dtype=torch.bfloat16, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind, B, Hkv", [("kv4", 3, 8), ("window", 2, 3)])
def test_attention_at_the_end_of_long_caches(kind, B, Hkv):
    """Slabs of 256 MB (4 bits) and 1 GB (bf16), the last of them past 2^32 bytes. What no row sees is never written."""
    rng = np.random.default_rng(1)
    n, win, sinks, D = 300, 150, 7, 128  # the first and the last n rows hold something
    x = Inputs(rng, B, 3, 2 * Hkv, Hkv, D, 2 * n, [2 * n - 3] * B, holes=0.1)
    ref, size, _ = x.reference(kind, win, sinks)
    x.upload(kind)
    long = [torch.empty(B, Hkv, CAP, t.shape[-1], dtype=t.dtype, device="cuda") for t in x.dcache]
    mask = torch.ones(B, CAP, dtype=torch.uint8, device="cuda")
    for big, small in zip(long, x.dcache):
        big[:, :, :n], big[:, :, CAP - n:] = small[:, :, :n], small[:, :, n:]
    mask[:, :n], mask[:, CAP - n:] = x.dmask[:, :n], x.dmask[:, n:]
    x.cap, x.dcache, x.dmask, x.dlen = CAP, long, mask, _i32([CAP] * B)
    out = torch.full((B, 3, 2 * Hkv, D), float("nan"), **BF)
    say(f"{kind} window over {CAP} rows")
    x.call(kind, win, sinks, out, x.workspace(kind, win, sinks))
    check(out, ref, size)


def test_kv4_attention_over_all_of_a_long_cache():
    """4194304 keys of which the mask leaves the first and the last few; the rest hold NaN."""
    rng = np.random.default_rng(2)
    n, D = 100, 64
    x = Inputs(rng, 1, 4, 4, 1, D, 2 * n, [2 * n - 4], holes=0.1)
    ref, size, _ = x.reference("kv4")
    x.upload("kv4")
    long = [torch.full((1, 1, CAP, t.shape[-1]), 255, dtype=torch.uint8, device="cuda") for t in x.dcache]
    mask = torch.zeros(1, CAP, dtype=torch.uint8, device="cuda")
    for big, small in zip(long, x.dcache):
        big[:, :, :n], big[:, :, CAP - n:] = small[:, :, :n], small[:, :, n:]
    mask[:, :n], mask[:, CAP - n:] = x.dmask[:, :n], x.dmask[:, n:]
    x.cap, x.dcache, x.dmask, x.dlen = CAP, long, mask, _i32([CAP])
    out = torch.full((1, 4, 4, D), float("nan"), **BF)
    say(f"kv4 over {CAP} rows")
    x.call("kv4", 0, 0, out, x.workspace("kv4", 0, 0))
    check(out, ref, size)


@pytest.mark.parametrize("rows", [5, 200])  # one workgroup per sequence, and blocks of rows
def test_kv4_append_at_the_end_of_long_caches(rows):
    import paper_2505_07680_amd as sr

    rng = np.random.default_rng(3)
    B, Hkv, D = 3, 8, 128
    k, v = (bf16(normal_bits(rng, (B, rows, Hkv, D))) for _ in range(2))
    gamma = _i32([rows - 1] * B)
    small, n1 = sr.Kv4Cache(B, Hkv, rows, D), _i32([0] * B)
    parts = ("k_codes", "k_powers", "v_codes", "v_powers")
    sr.specrouter_kv4_append(k, v, gamma, *(getattr(small, p) for p in parts), None, n1)
    long, n2 = sr.Kv4Cache(B, Hkv, CAP, D), _i32([CAP - rows] * B)
    say(f"append of {rows} rows at {CAP - rows}")
    sr.specrouter_kv4_append(k, v, gamma, *(getattr(long, p) for p in parts), None, n2)
    assert n2.tolist() == [CAP] * B
    for p in parts:
        assert torch.equal(getattr(long, p)[:, :, CAP - rows:], getattr(small, p)), p
        assert not getattr(long, p)[:, :, :CAP - rows].any(), p


def test_norm_rope_of_more_than_2_31_elements():
    import paper_2505_07680_amd as sr

    torch.manual_seed(4)
    B, rows, Hq, Hkv, D = 2, 70000, 120, 8, 128
    q, k = torch.randn(B, rows, Hq, D, **BF), torch.randn(B, rows, Hkv, D, **BF)
    assert q.numel() > 1 << 31
    w, table = torch.rand(D, **BF) + 0.5, sr.rope_table(rows + 10, D)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pos, gamma = _i32([3, 9]), _i32([rows - 1] * 2)
    say(f"norm and rotation of {q.numel()} elements")
    sr.specrouter_qk_norm_rope(q, k, w, w, 1e-6, table, pos, gamma, qo, ko)
    at, m = rows - 50, 50  # the last rows of each sequence in a call of their own
    q1, k1 = q[:, at:].contiguous(), k[:, at:].contiguous()
    qr, kr = torch.empty_like(q1), torch.empty_like(k1)
    sr.specrouter_qk_norm_rope(q1, k1, w, w, 1e-6, table, pos + at, _i32([m - 1] * 2), qr, kr)
    assert torch.equal(qo[:, at:].view(torch.int16), qr.view(torch.int16))
    assert torch.equal(ko[:, at:].view(torch.int16), kr.view(torch.int16))
