"""The calls around a verifier's attention as a serving loop makes them, several
steps in a row on the device: queries and keys normed and rotated, the rows
appended to a 4-bit (or bf16) cache, attention over it with or without a
window, drafts accepted and lengths rolled back -- each step's outputs against
the reference on what the device then holds."""

import numpy as np
import pytest
import torch

import oracle
from oracle import kv4, rope, window
from workloads import level_inputs, small_shape

from gpu_util import dev, host
from operator_util import bf16, check, normal_bits, say

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def _bits(t):
    return host(t.contiguous().view(torch.int16)).view(np.uint16)


def _rope_close(got, want, size):
    """The rotation's output, rounded once to bf16 (2^-8 of the value) from 32-bit arithmetic."""
    err = np.abs(host(got.float()) - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size + 1e-40).all()


@pytest.mark.parametrize("four,win,sinks", [(True, 0, 0), (True, 48, 4), (False, 48, 4)])
def test_prompt_and_verify_steps(four, win, sinks):
    import paper_2505_07680_amd as sr

    B, Hq, Hkv, D, L_cap, G, V = 4, 8, 2, 128, 260, 4, 1000
    rng = np.random.default_rng(int(four) + win)
    scale = D ** -0.5
    wq, wk = (torch.from_numpy(rng.normal(1, 0.2, D).astype(np.float32)).to(torch.bfloat16).cuda() for _ in range(2))
    table = sr.rope_table(L_cap, D)
    i32 = dict(dtype=torch.int32, device="cuda")
    length, status, phys = torch.zeros(B, **i32), torch.zeros(1, **i32), torch.zeros(1, **i32)
    mask = torch.zeros(B, L_cap, dtype=torch.uint8, device="cuda")
    if four:
        c = sr.Kv4Cache(B, Hkv, L_cap, D)
        cache = [c.k_codes, c.k_powers, c.v_codes, c.v_powers]
    else:
        cache = [torch.zeros(B, Hkv, L_cap, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def rows(n, gamma):
        """One projection of n new rows, normed, rotated and appended: (q, q bits)."""
        x = bf16(normal_bits(rng, (B, n, (Hq + 2 * Hkv) * D)))
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], -1)
        q, k, v = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (Hkv, D)), v.unflatten(-1, (Hkv, D))
        qo, ko = (torch.zeros(B, n, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv))
        before = host(length).copy()
        pos = length.clone()
        sr.specrouter_qk_norm_rope(q, k, wq, wk, EPS, table, pos, gamma, qo, ko, status=status)
        old = [host(t if four else t.view(torch.int16)).copy() for t in cache]
        if four:
            sr.specrouter_kv4_append(ko, v, gamma, *cache, mask, length, status=status)
        else:
            sr.specrouter_kv_append(ko, v.contiguous(), gamma, *cache, mask, length, status=status)
        torch.cuda.synchronize()
        g = host(gamma)
        for got, src, w in ((qo, q, wq), (ko, k, wk)):
            want, live, size, st = rope.norm_rope(host(src.float()), host(w.float()), EPS, host(table), before, g)
            assert st == 0
            _rope_close(got[torch.from_numpy(live).cuda()], want[live], size[live])
        if four:
            new, _, kl, _, _, st = kv4.append(old, None, before, _bits(ko), _bits(v), g)
            assert st == 0
            for a, b in zip(cache, new):
                np.testing.assert_array_equal(host(a), b)
        else:
            kl = before + g + 1
        np.testing.assert_array_equal(host(length), kl)
        return qo

    if four:
        rows(100, dev(np.array([99, 80, 0, 50], np.int32)))  # prompts
    else:  # (specrouter_kv_append takes 17 rows at most)
        for _ in range(6):
            rows(17, dev(np.array([16, 12, 0, 8], np.int32)))
    call = sr.specrouter_verify_attention_kv4 if four else sr.specrouter_verify_attention_window
    make = sr.attention_kv4_workspace if four else sr.attention_window_workspace
    ws = make(B, G, Hq, Hkv, D, L_cap, win, sinks)
    acc = sr.AcceptBuffers(B, G, V, sr.SR_F32)
    for step in range(5):
        gamma = rng.integers(0, G + 1, B).astype(np.int32)
        gd = dev(gamma)
        q = rows(G + 1, gd)
        out = torch.empty(B, G + 1, Hq, D, dtype=torch.bfloat16, device="cuda")
        call(q, *cache, mask, length, gd, out, scale, win, sinks, ws, status)
        torch.cuda.synchronize()
        if four:
            h = [host(t) for t in cache]
            k, v = kv4.values(*h[:2]), kv4.values(*h[2:])
        else:
            k, v = (_bits(t) for t in cache)
        ref, size, st = window.verify_attention(_bits(q), k, v, host(length), gamma, scale, host(mask), win, sinks)
        assert st == 0
        check(out, ref, size)
        inp = level_inputs(small_shape(name=f"together-{step}", B=B, V=V, gamma=G, seed=50 + step), kv=False)
        kv = host(length).copy()
        kept = length.clone()
        sr.specrouter_accept_and_rollback(dev(inp.p_logits), dev(inp.q_logits), dev(inp.drafts), gd, dev(inp.u_acc),
                                          dev(inp.u_res), kept, acc.accept_len, acc.out_tokens, acc.new_len,
                                          acc.accept_prob, acc.p_tok, acc.q_tok, acc.kl, acc.tv, length, mask, phys,
                                          acc.workspace, status)
        torch.cuda.synchronize()
        want = oracle.accept_and_diverge(inp.p_logits, inp.q_logits, inp.drafts, gamma, inp.u_acc, inp.u_res, kv_len=kv)
        for b in range(B):
            if not want["boundary"][b]:
                assert int(acc.accept_len[b]) == want["accept_len"][b] and int(length[b]) == want["new_len"][b]
        m = host(mask)
        for b in range(B):
            n = int(length[b])
            assert (m[b, :n] == 1).all() and (m[b, n:] == 0).all()
        say(f"together four={four} window={win} step {step}: lengths {host(length).tolist()}")
    assert int(status) == 0
