"""specrouter_qk_norm_rope where queries and keys are made of the same rows, one of the two in place."""

import numpy as np
import pytest
import torch

from gpu_util import dev
from test_gpu_rope import EPS, _library, say  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,G1,H,Hk,D", [(1, 1, 4, 4, 64), (3, 5, 40, 40, 128), (2, 400, 24, 24, 128), (2, 300, 32, 5, 64)])
def test_one_of_the_two_in_place(B, G1, H, Hk, D, interleaved):
    """Heads of one row lie in several waves: none may read what another has already turned."""
    import paper_2505_07680_amd as sr

    rng = np.random.default_rng(H)
    x = torch.from_numpy(rng.normal(size=(B, G1, H, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    wq, wk = (torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda() for _ in range(2))
    table = sr.rope_table(G1 + 50, D)
    pos, gam = dev(np.arange(B, dtype=np.int32) * 7), dev(np.full(B, G1 - 1, np.int32))

    def call(q, k, q_out, k_out):
        sr.specrouter_qk_norm_rope(q, k, wq, wk, EPS, table, pos, gam, q_out, k_out, interleaved=interleaved)

    want_q, want_k = torch.empty_like(x), torch.empty_like(x[:, :, :Hk].contiguous())
    call(x, x[:, :, :Hk], want_q, want_k)
    for _ in range(4):
        say(f"rope shared rows B={B} rows={G1} H={H},{Hk} D={D}: queries in place")
        a, k_out = x.clone(), torch.zeros_like(want_k)
        call(a, a[:, :, :Hk], a, k_out)
        assert torch.equal(a, want_q) and torch.equal(k_out, want_k)
        if Hk == H:
            say(f"rope shared rows B={B} rows={G1} H={H},{Hk} D={D}: keys in place")
            a, q_out = x.clone(), torch.zeros_like(want_q)
            call(a, a, q_out, a)
            assert torch.equal(a, want_k) and torch.equal(q_out, want_q)
    a, k_out = x.clone(), torch.zeros_like(want_k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(a, a[:, :, :Hk], a, k_out)
    for _ in range(3):
        a.copy_(x), k_out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want_q) and torch.equal(k_out, want_k)
