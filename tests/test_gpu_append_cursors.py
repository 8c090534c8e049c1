"""A shared cursor outside the cache, up to the largest 32-bit value, leaves the caches of
both appends as they were and is flagged."""

import numpy as np
import pytest
import torch

from gpu_util import dev, host

pytestmark = pytest.mark.gpu
ST_KVLEN = 2


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("cursor", [-1, -2 ** 31, 61, 64, 2 ** 31 - 1, 2 ** 31 - 4, 2 ** 31 - 5])
@pytest.mark.parametrize("rows", [4, 60])
def test_cursor_outside_the_cache(cursor, rows):
    import paper_2505_07680_amd as sr

    B, Hkv, D, L = 3, 8, 128, 64
    new = [torch.randn(B, rows, Hkv, D, device="cuda").to(torch.bfloat16) for _ in range(2)]
    gamma = dev(np.full(B, rows - 1, np.int32))
    shared = torch.tensor([cursor], dtype=torch.int32, device="cuda")
    caches = {"bf16": [torch.randn(B, Hkv, L, D, device="cuda").to(torch.bfloat16) for _ in range(2)],
              "4 bits": [torch.randint(0, 256, (B, Hkv, L, n), dtype=torch.uint8, device="cuda")
                         for n in (D // 2, D // 32, D // 2, D // 32)]}
    for kind, cache in caches.items():
        if kind == "bf16" and rows > 17:
            continue
        print(f"[gpu-test] append {kind} rows={rows} cursor={cursor}", flush=True)
        mask = torch.zeros(B, L, dtype=torch.uint8, device="cuda")
        length = dev(np.array([0, 5, 1], np.int32))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        before = [t.clone() for t in cache]
        call = sr.specrouter_kv_append if kind == "bf16" else sr.specrouter_kv4_append
        call(*new, gamma, *cache, mask, length, shared_len=shared, status=status)
        torch.cuda.synchronize()
        assert int(status) == ST_KVLEN
        assert host(length).tolist() == [0, 5, 1] and int(mask.sum()) == 0
        for got, want in zip(cache, before):
            assert torch.equal(got, want)
