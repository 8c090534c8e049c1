"""GPU parity of the attention with a window and sinks over a bf16 cache
(specrouter_verify_attention_window) and over a 4-bit cache
(specrouter_verify_attention_kv4, with and without a window) against the fp64
reference."""

import numpy as np
import pytest
import torch

from oracle import kv4

from gpu_util import dev, host
from operator_util import Inputs, bf16_bits, check, say, tolerance

pytestmark = pytest.mark.gpu

KINDS = ["window", "kv4"]
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _library():
    import paper_2505_07680_amd as sr

    sr.load()
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("win", [1, 2, 15, 16, 17, 31, 33, 64, 100, 1000])
def test_windows(kind, win):
    """Every edge of a window against the tiles, with sinks before, at and past its first key."""
    rng = np.random.default_rng(win)
    x = Inputs(rng, 6, 4, 8, 2, 128, 300, [0, 1, 30, 97, 200, 296], [0, 3, 3, 1, 3, 3])
    for sinks in (0, 1, 4, 16, 33, 250):
        say(f"{kind} window={win} sinks={sinks}")
        x.compare(kind, win, sinks)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("Hq,Hkv,D,G1", [(1, 1, 64, 1), (4, 4, 64, 5), (8, 2, 128, 1), (16, 2, 64, 6), (32, 8, 128, 6),
                                         (8, 1, 128, 9), (12, 2, 64, 9), (16, 1, 128, 9), (5, 1, 128, 13),
                                         (16, 1, 64, 17)])
def test_heads_and_rows(kind, dtype, Hq, Hkv, D, G1):
    """1 to 272 query rows a kv head: every number of row blocks and query chunks."""
    rng = np.random.default_rng(Hq * G1)
    B = 3
    gamma = [G1 - 1, 0, (G1 - 1) // 2]
    x = Inputs(rng, B, G1, Hq, Hkv, D, 400, [37, 0, 383], gamma, holes=0.1)
    say(f"{kind} Hq={Hq} Hkv={Hkv} D={D} G1={G1}")
    x.compare(kind, 70, 5, DTYPES[dtype])
    if kind == "kv4":
        x.compare(kind, 0, 0, DTYPES[dtype])


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 511, 1000])
def test_kv4_lengths(L):
    """Lengths around the tiles and the splits, a cache that ends inside a tile, one row."""
    rng = np.random.default_rng(L)
    for D, Hq, Hkv in ((64, 4, 4), (128, 8, 2)):
        say(f"kv4 L={L} D={D}")
        Inputs(rng, 2, 1, Hq, Hkv, D, L, [L - 1, (L - 1) // 2]).compare("kv4")


@pytest.mark.parametrize("kind", KINDS)
def test_window_over_the_whole_cache_hides_nothing(kind):
    """From L_cap on a larger window changes no bit of the output, which is that of the
    call without a window: bit for bit over 4 bits, and over bf16, where that call sums in
    another order, as near as two results within the tolerance of one value are."""
    import paper_2505_07680_amd as sr

    rng = np.random.default_rng(3)
    x = Inputs(rng, 5, 6, 32, 8, 128, 500, rng.integers(0, 494, 5), rng.integers(0, 6, 5), holes=0.05)
    out, _ = x.run(kind, 500, 7, torch.float32)
    more, _ = x.run(kind, 2 ** 31 - 1, 2 ** 31 - 1, torch.float32)
    assert torch.equal(out, more)
    if kind == "window":
        want = torch.empty_like(out)
        sr.specrouter_verify_attention(x.dq, *x.dcache, x.dmask, x.dlen, x.dgam, want, x.scale,
                                       sr.attention_workspace(5, 5, 32, 8, 128, 500))
        torch.cuda.synchronize()
        ref, size, _ = x.reference(kind)
        check(want, ref, size)
        check(out, ref, size)
        assert (host(out - want) <= 2 * tolerance(ref, size, False)).all()
    else:
        want, _ = x.run(kind, 0, 0, torch.float32)
        assert torch.equal(out, want)


def test_bf16_output_is_the_fp32_output_rounded():
    rng = np.random.default_rng(4)
    for kind in KINDS:
        x = Inputs(rng, 3, 3, 8, 2, 64, 700, [697, 20, 300], holes=0.02)
        a, _ = x.run(kind, 100, 4, torch.float32)
        b, _ = x.run(kind, 100, 4, torch.bfloat16)
        assert torch.equal(a.to(torch.bfloat16), b)


@pytest.mark.parametrize("kind", KINDS)
def test_masks_that_leave_rows_empty(kind):
    rng = np.random.default_rng(5)
    x = Inputs(rng, 5, 4, 8, 2, 128, 260, [200, 200, 200, 255, 3], holes=0.0)
    x.mask[0] = 0                # nothing at all
    x.mask[1, 60:] = 0           # only keys before the window, and the sinks
    x.mask[2, :203] = 0          # only the last row's own key
    x.mask[3, 10:] = 0
    x.mask[4, :4] = 0            # rows 1 to 3 see only new keys
    x.mask[1] *= 7               # any non-zero byte is valid
    for win, sinks in ((64, 0), (64, 8), (1, 1)):
        x.compare(kind, win, sinks)
    if kind == "kv4":
        x.compare(kind)


@pytest.mark.parametrize("kind", KINDS)
def test_entries_that_no_row_sees_are_ignored(kind):
    """NaN and infinities between the sinks and the window, under the mask and past the length."""
    rng = np.random.default_rng(6)
    x = Inputs(rng, 3, 3, 8, 2, 64, 300, [290, 100, 5], holes=0.1)
    win, sinks = 50, 5
    ref, size, _ = x.reference(kind, win, sinks)
    for b in range(3):
        L, n = int(x.kv_len[b]), int(x.gamma[b]) + 1
        unseen = np.ones(300, bool)
        unseen[max(0, L - n - win + 1):L] = False
        unseen[:min(sinks, L)] = False
        unseen |= x.mask[b] == 0
        if kind == "window":
            x.k[b][:, unseen] = 0x7FC0
            x.v[b][:, unseen] = 0x7F80
        else:
            x.cache4[1][b][:, unseen] = 255
            x.cache4[3][b][:, unseen] = 255
    out, st = x.run(kind, win, sinks)
    assert st == 0
    check(out, ref, size)


def test_kv4_nan_groups_reach_the_rows_that_see_them():
    """A power of 255 in K makes the rows that see the key NaN; in V, the group's 32 columns."""
    rng = np.random.default_rng(7)
    for D in (64, 128):
        x = Inputs(rng, 2, 1, 4, 2, D, 100, [80, 80])
        x.cache4[1][0, 0, 40, 1] = 255
        x.cache4[3][1, 1, 60, 0] = 255
        out = host(x.run("kv4", dtype=torch.float32)[0])
        assert np.isnan(out[0, 0, :2]).all() and np.isfinite(out[0, 0, 2:]).all()
        assert np.isnan(out[1, 0, 2:, :32]).all() and np.isfinite(out[1, 0, 2:, 32:]).all()
        assert np.isfinite(out[1, 0, :2]).all()


def test_kv4_small_and_large_powers():
    """Values from 2^-30 to 2^30 in one row's groups; the products take them exactly."""
    rng = np.random.default_rng(8)
    x = Inputs(rng, 2, 2, 4, 2, 128, 200, [150, 198])
    x.cache4[1][:] = rng.integers(97, 128, x.cache4[1].shape)
    x.cache4[3][:] = rng.integers(97, 158, x.cache4[3].shape)
    x.compare("kv4", dtype=torch.float32)
    x.compare("kv4", 77, 3, dtype=torch.float32)


@pytest.mark.parametrize("kind", KINDS)
def test_rising_and_falling_scores(kind):
    """Scores far apart along the cache: the softmax reference has to follow them."""
    rng = np.random.default_rng(9)
    for sign in (1, -1):
        x = Inputs(rng, 2, 2, 4, 1, 64, 600, [598, 300], four=True)
        ramp = np.linspace(-3, 3, 600)[::sign]
        u = rng.normal(size=64)
        u /= np.linalg.norm(u)
        x.q[:] = bf16_bits(np.broadcast_to(10 * u, x.q.shape))
        x.k[:] = bf16_bits(np.broadcast_to(ramp[None, None, :, None] * u * 3, x.k.shape) + rng.normal(0, 0.05, x.k.shape))
        x.cache4[0], x.cache4[1] = kv4.to_4_bits(x.k)
        x.compare(kind, 600 if kind == "window" else 0, 0, torch.float32)


@pytest.mark.parametrize("kind", KINDS)
def test_bad_sequences_are_flagged_and_zero(kind):
    rng = np.random.default_rng(10)
    x = Inputs(rng, 6, 4, 4, 2, 64, 100, [90] * 6)
    x.gamma[1], x.gamma[2] = 4, -1
    x.kv_len[3], x.kv_len[4], x.kv_len[5] = 101, 3, -7
    out, st = x.run(kind, 20, 2)
    ref, size, rst = x.reference(kind, 20, 2)
    assert st == rst == 3
    check(out, ref, size)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,Hq,Hkv,D,G1,cap,win", [(1, 8, 2, 128, 2, 9000, 3000), (1, 4, 4, 64, 5, 5000, 5000),
                                                   (150, 16, 8, 64, 3, 260, 120), (70, 32, 32, 128, 1, 200, 64),
                                                   (40, 64, 8, 128, 9, 300, 150), (3, 64, 8, 128, 9, 2500, 2000)])
def test_splits_and_dispatch_order(kind, B, Hq, Hkv, D, G1, cap, win):
    """One long sequence in many splits, more workgroups than fit at once, several query chunks."""
    rng = np.random.default_rng(B)
    gamma = rng.integers(0, G1, B)
    ctx = rng.integers(0, cap - G1 + 1, B)
    ctx[0], gamma[0] = cap - G1, G1 - 1
    x = Inputs(rng, B, G1, Hq, Hkv, D, cap, ctx, gamma, holes=0.02 if B % 2 else None)
    say(f"{kind} B={B} {Hq}/{Hkv}x{D} cap={cap}")
    x.compare(kind, win, 4)
    if kind == "kv4":
        x.compare(kind)


@pytest.mark.parametrize("kind", KINDS)
def test_workspace_is_reused_and_runs_repeat(kind):
    """One workspace, the calls in a row, captured and replayed, on another stream: the same bits."""
    rng = np.random.default_rng(12)
    x = Inputs(rng, 3, 3, 16, 2, 128, 3000, [2990, 40, 1500])
    win, sinks = 2000, 4
    x.upload(kind)
    ws = x.workspace(kind, win, sinks)
    assert ws is not None
    shape = (x.B, x.G1, x.Hq, x.D)
    first = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    x.call(kind, win, sinks, first, ws)
    torch.cuda.synchronize()
    ref, size, _ = x.reference(kind, win, sinks)
    check(first, ref, size)
    out = torch.empty_like(first)
    for _ in range(3):
        out.fill_(float("nan"))
        x.call(kind, win, sinks, out, ws)
        assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.call(kind, win, sinks, out, ws)
    for n in range(4):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        if n == 1:  # shorter sequences, then the first lengths again, by way of the same buffers
            x.dlen.copy_(dev(np.array([200, 43, 7], np.int32)))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.isfinite(out).all()
            x.dlen.copy_(dev(x.kv_len))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.fill_(float("nan"))
        x.call(kind, win, sinks, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, first)


def test_two_calls_at_once_on_two_streams():
    rng = np.random.default_rng(13)
    xs = [Inputs(rng, 2, 2, 8, 2, 128, 4000, [3990, 1000]) for _ in range(2)]
    kinds = ["window", "kv4"]
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for x, kind in zip(xs, kinds):
        x.upload(kind)
        x.ws = x.workspace(kind, 3500, 4)
        outs.append(torch.empty((x.B, x.G1, x.Hq, x.D), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, kind, out, s in zip(xs, kinds, outs, streams):
            with torch.cuda.stream(s):
                x.call(kind, 3500, 4, out, x.ws)
    torch.cuda.synchronize()
    for x, kind, out in zip(xs, kinds, outs):
        ref, size, _ = x.reference(kind, 3500, 4)
        check(out, ref, size)


@pytest.mark.parametrize("kind", KINDS)
def test_binding_refuses_what_does_not_fit(kind):
    rng = np.random.default_rng(14)
    x = Inputs(rng, 2, 3, 4, 2, 64, 2000, [50, 60])
    x.upload(kind)
    good = torch.empty((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    ws = x.workspace(kind, 64, 0)
    x.call(kind, 64, 0, good, ws)
    with pytest.raises(RuntimeError):
        x.call(kind, -1, 0, good, ws)
    with pytest.raises(RuntimeError):
        x.call(kind, 64, -1, good, ws)
    if kind == "window":
        with pytest.raises(RuntimeError):
            x.call(kind, 0, 0, good, ws)
    big = x.workspace(kind, 2000, 0)
    assert big is not None
    with pytest.raises(RuntimeError):
        x.call(kind, 2000, 0, good, None)
    with pytest.raises(RuntimeError):
        x.call(kind, 2000, 0, good, big[:64])
    for out in (good.half(), good[:, :2], good.cpu(), good.transpose(1, 2)):
        with pytest.raises((ValueError, TypeError)):
            x.call(kind, 64, 0, out, ws)
    for name, value in (("dq", x.dq.float()), ("dq", x.dq[:, :, :2]), ("dlen", x.dlen.long()), ("dgam", x.dgam[:1]),
                        ("dmask", torch.ones(2, 1999, dtype=torch.uint8, device="cuda")),
                        ("dcache", [t[:, :1] for t in x.dcache]), ("dcache", [t[..., :16] for t in x.dcache])):
        keep = getattr(x, name)
        setattr(x, name, value)
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            x.call(kind, 64, 0, good, ws)
        setattr(x, name, keep)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_nan_keys_reach_the_output_through_every_merge(kind, D):
    """A sequence split many ways: rows whose only visible keys are NaN, or some of whose
    splits hold nothing but a NaN key, are NaN; a row that sees no key stays 0."""
    rng = np.random.default_rng(15)
    cap = 20000
    x = Inputs(rng, 1, 2, 4, 2, D, cap, [19000], holes=0.0)
    for at, nan in (([700], [700]), ([700, 15000], [700]), ([700, 701, 9000, 18999], [700, 9000]), (range(0, 19000, 37), [37])):
        x.mask[:] = 0
        x.mask[0, list(at)] = 1
        k, p = x.k.copy(), x.cache4[1].copy()
        x.k[0, 0, nan] = 0x7FC0
        x.cache4[1][0, 0, nan] = 255
        out = host(x.run(kind, cap, 0, dtype=torch.float32)[0])
        x.k, x.cache4[1] = k, p
        say(f"{kind} D={D} visible {len(list(at))}")
        assert np.isnan(out[0, :, :2]).all()
        assert np.isfinite(out[0, :, 2:]).all() and (out[0, :, 2:] != 0).any()
    x.mask[:] = 0
    x.k[0, 0] = 0x7FC0
    x.cache4[1][0, 0] = 255
    assert (host(x.run(kind, cap, 0, dtype=torch.float32)[0]) == 0).all()


@pytest.mark.parametrize("B,Hq,Hkv,D,G1,cap,win", [
    (2, 64, 8, 128, 8, 10000, 9600),  # two groups of two row blocks
    (2, 64, 8, 64, 9, 10000, 9600),   # of three
    (1, 24, 2, 128, 16, 40000, 39000),  # two chunks of them
    (1, 24, 2, 64, 16, 40000, 39000),
    (40, 64, 8, 64, 9, 700, 300),     # chunks of two row blocks, in order
    (33, 64, 8, 64, 12, 700, 600),    # of three, not ordered
    (3, 32, 1, 64, 10, 500, 300),     # seven chunks
])
def test_forms_of_many_rows(B, Hq, Hkv, D, G1, cap, win):
    rng = np.random.default_rng(16)
    ctx = rng.integers(cap - cap // 4, cap - G1, B)
    gamma = rng.integers(0, G1, B).astype(np.int32)
    gamma[0] = G1 - 1
    x = Inputs(rng, B, G1, Hq, Hkv, D, cap, ctx, gamma=gamma, holes=0.05, four=False)
    say(f"B={B} rows={Hq // Hkv * G1} D={D} window={win}")
    x.compare("window", win, 5)


@pytest.mark.parametrize("B,Hq,Hkv,D,G1,cap,win", [(2, 4, 4, 64, 2, 3000, 0), (17, 8, 2, 64, 3, 1500, 0), (64, 4, 4, 64, 1, 700, 0),
                                                   (65, 4, 2, 64, 1, 700, 0), (63, 3, 3, 128, 2, 600, 0), (30, 12, 3, 64, 17, 500, 0),
                                                   (9, 8, 1, 128, 5, 5000, 0), (20, 6, 3, 64, 4, 2500, 900), (1, 4, 2, 64, 3, 20000, 0)])
def test_kv4_batches_dealt_by_their_lengths(B, Hq, Hkv, D, G1, cap, win):
    """One long sequence among short ones, all alike, and bad ones in between, over one workspace."""
    rng = np.random.default_rng(17)
    x = Inputs(rng, B, G1, Hq, Hkv, D, cap, [cap - G1] * B, holes=0.03)
    x.upload("kv4")
    ws = x.workspace("kv4", win, 4)
    for lengths in ("alike", "one long", "ragged", "bad"):
        x.gamma[:] = rng.integers(0, G1, B)
        low = rng.integers(0, 40, B)
        ctx = {"alike": np.full(B, cap - G1), "one long": low, "ragged": rng.integers(0, cap - G1 + 1, B), "bad": low}[lengths]
        ctx[B // 2] = cap - G1
        x.kv_len[:] = ctx + x.gamma + 1
        if lengths == "bad":
            x.gamma[::3] = G1
            x.kv_len[1::5] = cap + 1
        x.dlen, x.dgam = dev(x.kv_len), dev(x.gamma)
        out = torch.full((B, G1, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        say(f"B={B} {Hq}/{Hkv}x{D} cap={cap} {lengths}")
        x.call("kv4", win, 4, out, ws, st)
        ref, size, rst = x.reference("kv4", win, 4)
        assert int(st) == rst
        check(out, ref, size)
