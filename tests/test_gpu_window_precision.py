"""How the attention with a window rounds its weights, against the attention without one.

Where that call's softmax references follow the tiles, or a wave has one tile, the
largest key of every tile has a weight that bf16 holds exactly. Here no two keys of any
tile count (the others lie 80 powers of two below), so that all weights are exact
and only 32-bit roundings are left."""

import numpy as np
import pytest
import torch

from gpu_util import host
from operator_util import Inputs, bf16_bits, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def _inputs(rng, B, Hq, Hkv, D, G1, L):
    x = Inputs(rng, B, G1, Hq, Hkv, D, L, [L - G1] * B, four=False)
    x.q[:] = 0
    x.q[..., 0] = bf16_bits(np.float32(1))
    score = np.full((B, Hkv, L), -60.0)
    at = np.arange(0, L - 127, 128)  # (two tiles of one softmax step lie 64 keys apart: one tile of every eight)
    for b in range(B):
        for g in range(Hkv):
            score[b, g, at + 16 * rng.integers(0, 8) + rng.integers(0, 16, len(at))] = rng.uniform(-3, 3, len(at))
    x.k[..., 0] = bf16_bits(score / x.scale)
    return x


@pytest.mark.parametrize("B,Hq,Hkv,D,G1,L", [
    (1, 32, 8, 128, 6, 4096),    # two row blocks
    (1, 4, 2, 64, 3, 4096),      # one
    (1, 8, 2, 64, 12, 4096),     # three
    (2, 64, 8, 128, 9, 2048),    # rows in two chunks
    (2, 64, 8, 64, 9, 1024),
    (1, 24, 2, 128, 16, 40000),  # two groups of rows, two chunks of them
    (1, 16, 2, 64, 8, 40000),    # two groups of two row blocks
])
def test_a_window_over_the_whole_cache_is_as_exact_as_none(B, Hq, Hkv, D, G1, L):
    """Tolerance: exponents up to 16 powers of two, each off by a few roundings of 2^-24
    (scale, reference, product), so weights by less than 2^-17; sums and rescalings of
    some hundred terms by 2^-24 each: 2^-16 of the average of |v| in all."""
    import paper_2505_07680_amd as sr

    x = _inputs(np.random.default_rng(L + Hq), B, Hq, Hkv, D, G1, L)
    ref, size, _ = x.reference("window")
    got = {"window": x.run("window", L, 0, torch.float32)[0]}
    got["none"] = torch.empty_like(got["window"])
    sr.specrouter_verify_attention(x.dq, *x.dcache, None, x.dlen, x.dgam, got["none"], x.scale,
                                   sr.attention_workspace(B, G1 - 1, Hq, Hkv, D, L))
    torch.cuda.synchronize()
    for kind in ("none", "window"):
        err = np.abs(host(got[kind]).astype(np.float64) - ref) / (size + 1e-30)
        say(f"{kind} B={B} {Hq}/{Hkv}x{D} rows={G1} L={L}: off by {err.max():.3g} of the average")
        assert (err <= 2.0 ** -16).all(), kind
