"""Both forms of specrouter_kv4_append, one workgroup per sequence and blocks of rows, at the
sizes where the choice between them changes: byte for byte against the reference."""

import numpy as np
import pytest

from oracle import kv4

from test_gpu_kv4_append import _library, _run, bf16, normal_bits, say  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [None, 3])
@pytest.mark.parametrize("B,G1,Hkv,D", [(1, 24, 8, 128), (1, 25, 8, 128), (2, 48, 8, 64), (2, 49, 8, 64), (5, 193, 1, 128),
                                        (5, 384, 1, 64), (129, 64, 8, 128), (140, 65, 8, 128), (200, 33, 31, 64),
                                        (256, 32, 8, 128), (257, 32, 8, 128), (300, 23, 8, 128)])
def test_sizes_around_the_choice(B, G1, Hkv, D, shared):
    """Full and ragged sequences, some with bad data, rows past gamma and other slots left as they were."""
    rng = np.random.default_rng(B + G1)
    L = G1 + 4
    gamma = rng.integers(0, G1, B)
    gamma[0] = G1 - 1
    kv_len = rng.integers(0, 4, B)
    want = 0
    if B > 100:
        gamma[7], kv_len[11], gamma[11] = G1, L, 1
        want = kv4.ST_GAMMA | (kv4.ST_KVLEN if shared is None else 0)
    say(f"kv4 append B={B} rows={G1} Hkv={Hkv} D={D} shared={shared}")
    kn, vn = (bf16(normal_bits(rng, (B, G1, Hkv, D))) for _ in range(2))
    assert _run(kn, vn, gamma, kv_len, L, shared, mask=B != 2, seen=B != 5) == want
