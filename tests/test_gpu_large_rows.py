"""Norm, rotation and the 4-bit append of calls too large for the caches: bit for
bit the results of the same rows in small calls (which the other tests hold
against the references), into a buffer of their own and in place."""

import pytest
import torch

pytestmark = pytest.mark.gpu
BF = dict(dtype=torch.bfloat16, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _same(a, b, what):
    assert torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16)), what


# bytes in and out of the whole call: 44 MB and 166 MB; of one sequence: up to 28 MB
@pytest.mark.parametrize("rows", [181, 677])
@pytest.mark.parametrize("D, interleaved", [(128, False), (128, True), (64, False), (64, True)])
def test_norm_rope(rows, D, interleaved):
    import paper_2505_07680_amd as sr

    torch.manual_seed(1)
    B, Hq, Hkv = 6, 5120 // D, 5120 // D
    q, k = torch.randn(B, rows, Hq, D, **BF), torch.randn(B, rows, Hkv, D, **BF)
    wq, wk = torch.rand(D, **BF) + 0.5, torch.rand(D, **BF) + 0.5
    table = sr.rope_table(2000, D // 2)
    pos, gamma = _i32([0, 5, 600, 1, 17, 2]), _i32([rows - 1, rows - 2, 0, rows - 1, rows // 2, rows - 1])
    args = dict(eps=1e-6, rope_table=table, interleaved=interleaved)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 9.0)
    sr.specrouter_qk_norm_rope(q, k, wq, wk, position=pos, gamma=gamma, q_out=qo, k_out=ko, **args)
    for b in range(B):
        print(f"[gpu-test] rope rows={rows} D={D} b={b}", flush=True)
        q1, k1 = torch.full_like(q[:1], 7.0), torch.full_like(k[:1], 9.0)
        sr.specrouter_qk_norm_rope(q[b:b + 1], k[b:b + 1], wq, wk, position=pos[b:b + 1], gamma=gamma[b:b + 1],
                                   q_out=q1, k_out=k1, **args)
        _same(qo[b:b + 1], q1, ("q", b))
        _same(ko[b:b + 1], k1, ("k", b))
    for b, g in enumerate(gamma.tolist()):
        q[b, g + 1:], k[b, g + 1:] = 7.0, 9.0
    sr.specrouter_qk_norm_rope(q, k, wq, wk, position=pos, gamma=gamma, q_out=q, k_out=k, **args)
    _same(q, qo, "q in place")
    _same(k, ko, "k in place")


# 49 MB and 164 MB; up to 33 MB
@pytest.mark.parametrize("rows", [601, 2003])
@pytest.mark.parametrize("D", [64, 128])
def test_kv4_append(rows, D):
    import paper_2505_07680_amd as sr

    torch.manual_seed(2)
    B, Hkv, L_cap = 5, 2048 // D, 2100
    k, v = torch.randn(B, rows, Hkv, D, **BF), torch.randn(B, rows, Hkv, D, **BF)
    gamma, start = _i32([rows - 1, rows - 2, 3, rows - 1, rows // 2]), [0, 9, 1000, 64, 5]
    big, kv_len = sr.Kv4Cache(B, Hkv, L_cap, D), _i32(start)
    parts = ("k_codes", "k_powers", "v_codes", "v_powers")
    ks, vs = torch.full_like(k, 7.0), torch.full_like(v, 9.0)
    sr.specrouter_kv4_append(k, v, gamma, *(getattr(big, p) for p in parts), None, kv_len, k_seen=ks, v_seen=vs)
    for b in range(B):
        print(f"[gpu-test] append rows={rows} D={D} b={b}", flush=True)
        one, n1 = sr.Kv4Cache(1, Hkv, L_cap, D), _i32(start[b:b + 1])
        k1, v1 = torch.full_like(k[:1], 7.0), torch.full_like(v[:1], 9.0)
        sr.specrouter_kv4_append(k[b:b + 1], v[b:b + 1], gamma[b:b + 1], *(getattr(one, p) for p in parts), None, n1,
                                 k_seen=k1, v_seen=v1)
        for p in parts:
            assert torch.equal(getattr(big, p)[b:b + 1], getattr(one, p)), (p, b)
        _same(ks[b:b + 1], k1, ("k", b))
        _same(vs[b:b + 1], v1, ("v", b))
        assert int(n1) == int(kv_len[b]) == start[b] + int(gamma[b]) + 1
    again, n2 = sr.Kv4Cache(B, Hkv, L_cap, D), _i32(start)
    for b, g in enumerate(gamma.tolist()):
        k[b, g + 1:], v[b, g + 1:] = 7.0, 9.0
    sr.specrouter_kv4_append(k, v, gamma, *(getattr(again, p) for p in parts), None, n2, k_seen=k, v_seen=v)
    _same(k, ks, "k in place")
    _same(v, vs, "v in place")
    for p in parts:
        assert torch.equal(getattr(again, p), getattr(big, p)), p
