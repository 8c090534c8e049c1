"""GPU parity of specrouter_kv4_append against the reference, byte for byte:
steps and prompts, own and shared cursors, views of one projection, every bf16
value, bad data, graph replay, refusals."""

import numpy as np
import pytest
import torch

from oracle import kv4

from gpu_util import dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def say(msg):
    print(f"[gpu-test] {msg}", flush=True)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).cuda().view(torch.bfloat16)


def bits(t):
    return host(t.contiguous().view(torch.int16)).view(np.uint16)


def normal_bits(rng, shape, sigma=1.0):
    return (rng.normal(0, sigma, shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _run(kn, vn, gamma, kv_len, L_cap, shared=None, mask=True, seen=True, seed=0):
    """kn, vn: device tensors [B, G1, Hkv, D]. The call and the reference on the same cache."""
    import paper_2505_07680_amd as sr

    B, G1, Hkv, D = kn.shape
    rng = np.random.default_rng(seed)
    cache = [rng.integers(0, 256, (B, Hkv, L_cap, w)).astype(np.uint8) for w in (D // 2, D // 32, D // 2, D // 32)]
    m = (rng.random((B, L_cap)) < 0.5).astype(np.uint8) if mask else None
    cd = [dev(t) for t in cache]
    md = None if m is None else dev(m)
    ld = dev(np.asarray(kv_len, np.int32))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ks, vs = (torch.full((B, G1, Hkv, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sl = None if shared is None else torch.tensor([shared], dtype=torch.int32, device="cuda")
    sr.specrouter_kv4_append(kn, vn, dev(np.asarray(gamma, np.int32)), *cd, md, ld, shared_len=sl,
                             k_seen=ks if seen else None, v_seen=vs if seen else None, status=st)
    torch.cuda.synchronize()
    out, rm, rl, rseen, wrote, rst = kv4.append(cache, m, kv_len, bits(kn), bits(vn), gamma, phys_len=shared)
    assert int(st) == rst
    np.testing.assert_array_equal(host(ld), rl)
    if m is not None:
        np.testing.assert_array_equal(host(md), rm)
    for got, want in zip(cd, out):
        np.testing.assert_array_equal(host(got), want)
    if seen:
        for got, want in ((ks, rseen[0]), (vs, rseen[1])):
            g = host(got.float())
            np.testing.assert_array_equal(g[wrote].astype(np.float64), want[wrote])
            assert (g[~wrote] == 5.0).all()
    return rst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shared", [None, 40])
def test_steps(D, shared):
    rng = np.random.default_rng(D)
    B, Hkv, G1, L = 9, 3, 6, 70
    kv_len = rng.integers(0, 60, B)
    gamma = rng.integers(0, G1, B)
    gamma[3], gamma[4] = G1, -1          # bad windows
    kv_len[5], gamma[5] = L - 1, 2       # no room at its own cursor
    kv_len[6] = L + 5                    # a length outside [0, L_cap]
    kv_len[7], gamma[7] = L - G1, G1 - 1  # the last rows
    say(f"kv4 append step D={D} shared={shared}")
    kn, vn = (bf16(normal_bits(rng, (B, G1, Hkv, D))) for _ in range(2))
    assert _run(kn, vn, gamma, kv_len, L, shared) == kv4.ST_GAMMA | kv4.ST_KVLEN


@pytest.mark.parametrize("B,G1,Hkv,D,L", [(1, 1, 1, 64, 1), (1, 1, 8, 128, 5), (3, 17, 32, 128, 40), (2, 129, 8, 128, 131),
                                          (2, 700, 2, 64, 701), (3, 333, 5, 64, 400), (1, 1024, 1, 128, 1024),
                                          (1, 1025, 1, 128, 1025)])
def test_sizes_up_to_prompts(B, G1, Hkv, D, L):
    """One workgroup per sequence up to 1024 rows of all heads, blocks of rows beyond."""
    rng = np.random.default_rng(G1)
    gamma = rng.integers(0, G1, B)
    gamma[0] = G1 - 1
    kv_len = np.zeros(B, np.int64)
    kv_len[B - 1] = min(2, L - G1)
    say(f"kv4 append B={B} rows={G1} Hkv={Hkv} D={D}")
    kn, vn = (bf16(normal_bits(rng, (B, G1, Hkv, D))) for _ in range(2))
    assert _run(kn, vn, gamma, kv_len, L, mask=G1 % 2 == 1, seen=G1 != 700) == 0


def test_bad_prompts_are_left_alone():
    rng = np.random.default_rng(2)
    B, G1, Hkv, D, L = 5, 300, 4, 64, 320
    kn, vn = (bf16(normal_bits(rng, (B, G1, Hkv, D))) for _ in range(2))
    assert _run(kn, vn, [299, 300, 50, 299, 0], [21, 0, -1, 20, 0], L) == kv4.ST_GAMMA | kv4.ST_KVLEN


def test_views_of_one_projection():
    rng = np.random.default_rng(3)
    B, G1, Hq, Hkv, D = 3, 5, 4, 2, 128
    x = bf16(normal_bits(rng, (B, G1, (Hq + 2 * Hkv) * D)))
    _, k, v = x.split([Hq * D, Hkv * D, Hkv * D], -1)
    assert _run(k.unflatten(-1, (Hkv, D)), v.unflatten(-1, (Hkv, D)), [4, 0, 2], [0, 3, 9], 20) == 0


def test_every_bf16_value_under_every_power():
    """All 65536 values, in groups whose largest element is their own largest, and below larger neighbours."""
    rng = np.random.default_rng(4)
    D = 128
    every = np.arange(65536, dtype=np.uint16).reshape(1, -1, 1, D)  # ascending: neighbours share a power
    mixed = rng.permutation(65536).astype(np.uint16).reshape(1, -1, 1, D)
    exps = rng.integers(0, 255, (1, 512, 1, D // 32)).repeat(32, -1)
    spread = ((rng.integers(0, 2, (1, 512, 1, D)) << 15) | (np.clip(exps - rng.integers(0, 6, (1, 512, 1, D)), 0, 254) << 7)
              | rng.integers(0, 128, (1, 512, 1, D))).astype(np.uint16)
    for name, a, b in (("every", every, mixed), ("spread", spread, spread[:, ::-1])):
        say(f"kv4 append values {name}")
        assert _run(bf16(a), bf16(b), [511], [0], 512) == 0


def test_graph_replays_and_another_stream():
    """Captured, the append runs on with each replay: the cursor is read on the device."""
    import paper_2505_07680_amd as sr

    rng = np.random.default_rng(6)
    B, G1, Hkv, D, L = 3, 2, 2, 64, 64
    for rows in (2, 600):  # the step form and the prompt form
        Lr = L if rows == 2 else 4 * rows
        kn, vn = (bf16(normal_bits(rng, (B, rows, Hkv, D))) for _ in range(2))
        gam = dev(np.array([rows - 1, 0, rows - 2], np.int32))
        kv = torch.zeros(B, dtype=torch.int32, device="cuda")
        cache = sr.Kv4Cache(B, Hkv, Lr, D)
        args = (cache.k_codes, cache.k_powers, cache.v_codes, cache.v_powers)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sr.specrouter_kv4_append(kn, vn, gam, *args, None, kv)
        assert host(kv).tolist() == [0, 0, 0]
        want = [np.zeros(t.shape, np.uint8) for t in args]
        length = np.zeros(B, np.int32)
        for _ in range(3):
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want, _, length, _, _, _ = kv4.append(want, None, length, bits(kn), bits(vn), host(gam))
            np.testing.assert_array_equal(host(kv), length)
            for got, w in zip(args, want):
                np.testing.assert_array_equal(host(got), w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            kv.zero_()
            sr.specrouter_kv4_append(kn, vn, gam, *args, None, kv)
        torch.cuda.current_stream().wait_stream(side)
        np.testing.assert_array_equal(host(kv), host(gam) + 1)


def test_binding_refuses_what_does_not_fit():
    import paper_2505_07680_amd as sr

    bf = dict(dtype=torch.bfloat16, device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    c = sr.Kv4Cache(2, 3, 10, 64)
    good = dict(k_new=torch.zeros(2, 4, 3, 64, **bf), v_new=torch.zeros(2, 4, 3, 64, **bf), gamma=i, k_codes=c.k_codes,
                k_powers=c.k_powers, v_codes=c.v_codes, v_powers=c.v_powers, cache_mask=None, kv_len=i.clone())
    sr.specrouter_kv4_append(**good)
    bad = [
        dict(k_new=torch.zeros(2, 4, 2, 64, **bf)), dict(k_new=good["k_new"].half()), dict(gamma=i.long()),
        dict(kv_len=i[:1]), dict(k_codes=c.k_codes[:, :, :9]), dict(k_codes=c.k_codes.to(torch.int8)),
        dict(v_powers=c.k_codes), dict(cache_mask=torch.zeros(2, 9, dtype=torch.uint8, device="cuda")),
        dict(cache_mask=torch.zeros(2, 10, dtype=torch.int32, device="cuda")), dict(shared_len=i),
        dict(k_seen=torch.zeros(2, 4, 3, 64, device="cuda")), dict(v_seen=torch.zeros(2, 3, 3, 64, **bf)),
        dict(kv_len=i.cpu()), dict(k_new=torch.zeros(2, 11, 3, 64, **bf), v_new=torch.zeros(2, 11, 3, 64, **bf)),
        dict(k_new=torch.zeros(2, 3, 4, 64, **bf).transpose(1, 2)),
    ]
    for change in bad:
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            sr.specrouter_kv4_append(**{**good, **change})
    torch.cuda.synchronize()
