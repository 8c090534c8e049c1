"""GPU parity of specrouter_verify_attention_window where its workgroups outnumber what the
device holds at once, with and without the table that gives them their jobs, longest first."""

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


@pytest.mark.parametrize("B,Hq,Hkv,D,G1,cap,win,chunks,table", [
    (200, 16, 4, 64, 5, 1050, 900, 1, True),
    (200, 16, 4, 64, 5, 1050, 500, 1, False),
    (100, 32, 4, 64, 9, 1050, 900, 2, True),
    (100, 32, 4, 64, 9, 600, 400, 2, False),
    (130, 16, 2, 64, 17, 1050, 900, 3, True),
    (200, 16, 2, 64, 17, 600, 300, 3, True),
    (130, 16, 2, 128, 17, 300, 60, 3, False),
])
def test_jobs_with_and_without_the_table(B, Hq, Hkv, D, G1, cap, win, chunks, table):
    """Ragged, alike, and with bad sequences in between, over one workspace."""
    rng = np.random.default_rng(B + win)
    x = Inputs(rng, B, G1, Hq, Hkv, D, cap, [0] * B, holes=0.02, four=False)
    x.upload("window")
    ws = x.workspace("window", win, 4)
    assert (0 if ws is None else ws.numel()) == (4 * B * Hkv * chunks if table else 0)  # (one split each)
    for lengths in ("ragged", "alike", "bad"):
        x.gamma[:] = rng.integers(0, G1, B)
        ctx = np.full(B, cap - G1) if lengths == "alike" else rng.integers(0, cap - G1 + 1, B)
        x.kv_len[:] = ctx + x.gamma + 1
        if lengths == "bad":
            x.gamma[::7] = G1
            x.kv_len[1::9] = cap + 1
        x.dlen, x.dgam = dev(x.kv_len), dev(x.gamma)
        out = torch.full((B, G1, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        say(f"window B={B} {Hq}/{Hkv}x{D} rows={G1} cap={cap} window={win} {lengths}")
        x.call("window", win, 4, out, ws, st)
        torch.cuda.synchronize()
        ref, size, rst = x.reference("window", win, 4)
        assert int(st) == rst
        check(out, ref, size)
