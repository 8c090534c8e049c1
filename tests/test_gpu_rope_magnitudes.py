"""GPU parity of specrouter_qk_norm_rope for heads whose squares leave the range of 32 bits."""

import numpy as np
import pytest
import torch

from gpu_util import dev
from test_gpu_rope import _check, _library, say  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

SIZES = [1e-39, 1e-36, 1e-30, 1e-22, 1e-19, 1e-15, 1e-9, 1.0, 1e9, 1e17, 1e18, 1e19, 1e22, 1e30, 1e37, 1.2e38]


@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-30, 1e-6, 1.0])
@pytest.mark.parametrize("D,weights,interleaved", [(64, "f32", False), (128, "bf16", True), (128, "f32", False)])
def test_heads_of_every_magnitude(D, weights, interleaved, eps):
    """Each head by its own norm, whatever its neighbours in a wave: sizes from bf16's
    subnormal numbers to its largest, one head of mixed sizes, keys without a norm unchanged in size."""
    import paper_2505_07680_amd as sr

    rng = np.random.default_rng(D)
    eps = float(np.float32(eps))
    sizes = rng.permutation(SIZES + [1.0])
    x = rng.uniform(0.5, 2.0, (1, 2, len(sizes), D)) * rng.choice([-1, 1], (1, 2, len(sizes), D))
    x *= sizes[None, None, :, None]
    x[:, :, -1, ::3] = 1e25
    q = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
    k = torch.from_numpy(x[:, :, :3].clip(-1e37, 1e37).astype(np.float32)).to(torch.bfloat16).cuda()
    w = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).to(torch.float32 if weights == "f32" else torch.bfloat16).cuda()
    table, pos, gamma = sr.rope_table(64, D), [11], [1]
    for wk in (None, w):
        qo, ko = torch.zeros_like(q), torch.zeros_like(k)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        say(f"rope D={D} eps={eps} weights={weights} keys normed={wk is not None}")
        sr.specrouter_qk_norm_rope(q, k, w, wk, eps, table, dev(np.asarray(pos, np.int32)),
                                   dev(np.asarray(gamma, np.int32)), qo, ko, interleaved=interleaved, status=st)
        torch.cuda.synchronize()
        assert _check(qo, torch.zeros_like(q), q, w, eps, table, pos, gamma, interleaved) == 0
        assert _check(ko, torch.zeros_like(k), k, wk, eps, table, pos, gamma, interleaved) == 0
        assert int(st) == 0
