"""GPU parity of specrouter_verify_attention_kv4 where its workgroups outnumber what the
device holds at once and caches are long: they take their jobs from a table, longest first."""

import numpy as np
import pytest
import torch

from gpu_util import dev
from operator_util import Inputs, check, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def _inputs(rng, B, G1, Hq, Hkv, D, cap):
    x = Inputs(rng, B, G1, Hq, Hkv, D, 8, [8 - G1 if G1 < 8 else 0] * B, four=False)  # (the bf16 cache is not used)
    x.cap = cap
    shape = lambda n: (B, Hkv, cap, n)
    x.cache4 = [rng.integers(0, 256, shape(D // 2)).astype(np.uint8), rng.integers(124, 128, shape(D // 32)).astype(np.uint8),
                rng.integers(0, 256, shape(D // 2)).astype(np.uint8), rng.integers(124, 128, shape(D // 32)).astype(np.uint8)]
    x.mask = (rng.random((B, cap)) >= 0.02).astype(np.uint8)
    return x


@pytest.mark.parametrize("B,Hq,Hkv,D,G1,splits,win,sinks", [
    (200, 16, 4, 64, 5, 1, 0, 0),   # two row blocks
    (200, 16, 4, 64, 5, 1, 1100, 4),
    (130, 8, 8, 64, 2, 1, 0, 0),    # one
    (130, 8, 8, 64, 2, 1, 1100, 4),
    (120, 64, 1, 64, 5, 1, 0, 0),   # seven query chunks
    (120, 64, 1, 64, 5, 1, 1100, 4),
    (100, 16, 1, 128, 9, 2, 0, 0),  # three of them, and two splits
    (180, 16, 1, 128, 9, 1, 1200, 40),
])
def test_jobs_from_the_table(B, Hq, Hkv, D, G1, splits, win, sinks):
    """Ragged, alike, and with bad sequences in between, over one workspace."""
    rng = np.random.default_rng(B)
    cap, R = 1300, Hq // Hkv * G1
    x = _inputs(rng, B, G1, Hq, Hkv, D, cap)
    jobs = B * Hkv * -(-R // 48) * splits
    x.upload("kv4")
    ws = x.workspace("kv4", win, sinks)
    partials = 0 if splits == 1 else 128 * jobs // splits + B * Hkv * splits * R * (D + 2) * 4
    assert ws is not None and ws.numel() == -(-partials // 16) * 16 + 4 * jobs  # (the table is there)
    for lengths in ("ragged", "alike", "bad", "short"):
        x.gamma[:] = rng.integers(0, G1, B)
        ctx = {"ragged": rng.integers(0, cap - G1 + 1, B), "alike": np.full(B, cap - G1),
               "bad": rng.integers(0, cap - G1 + 1, B), "short": rng.integers(0, 40, B)}[lengths]
        x.kv_len[:] = ctx + x.gamma + 1
        if lengths == "bad":
            x.gamma[::7] = G1
            x.kv_len[1::9] = cap + 1
            x.kv_len[2::11] = 0
        x.dlen, x.dgam = dev(x.kv_len), dev(x.gamma)
        out = torch.full((B, G1, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        say(f"kv4 table B={B} {Hq}/{Hkv}x{D} rows={G1} window={win} {lengths}")
        x.call("kv4", win, sinks, out, ws, st)
        torch.cuda.synchronize()
        ref, size, rst = x.reference("kv4", win, sinks)
        assert int(st) == rst
        check(out, ref, size)
