"""Helpers of the GPU tests of the windowed and the 4-bit attention."""

from __future__ import annotations

import numpy as np
import torch

from oracle import kv4, window

from gpu_util import dev, host


def say(msg):
    print(f"[gpu-test] {msg}", flush=True)


def bf16_bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def normal_bits(rng, shape, sigma=1.0):
    return bf16_bits(rng.normal(0, sigma, shape))


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def tolerance(ref, size, out_bf16):
    """Of an attention output: the weights are rounded to bf16, each off by at most
    2^-8 of itself, so their sum by 2^-8 of the same average of |v| (`size`); the
    scores' and sums' 32-bit roundings are less than a sixteenth of that for the
    values here (128 products of 2^-24, scores below 100). A bf16 output adds 2^-8
    of the value."""
    return 2.0 ** -8 * (1 + 1 / 16) * size + (2.0 ** -8 * np.abs(ref) if out_bf16 else 0.0) + 1e-30


def check(got, ref, size):
    out = host(got.float()).astype(np.float64)
    assert np.isfinite(out).all(), "output that is not finite"
    tol = tolerance(ref, size, got.dtype == torch.bfloat16)
    err = np.abs(out - ref)
    assert (err <= tol).all(), f"{(err > tol).sum()} outside, worst {np.max(err / tol):.3g} of the tolerance"
    assert (out[size.sum(-1) == 0] == 0).all()


class Inputs:
    """Random inputs of an attention call over a bf16 and a 4-bit cache that hold the same values."""

    def __init__(self, rng, B, G1, Hq, Hkv, D, cap, ctx, gamma=None, holes=None, sigma=1.0, four=True):
        self.B, self.G1, self.Hq, self.Hkv, self.D, self.cap = B, G1, Hq, Hkv, D, cap
        self.q = normal_bits(rng, (B, G1, Hq, D), sigma)
        self.k, self.v = (normal_bits(rng, (B, Hkv, cap, D)) for _ in range(2))
        self.four = four
        if four:  # codes and powers of these values' sizes
            self.cache4 = [rng.integers(0, 256, (B, Hkv, cap, D // 2)).astype(np.uint8),
                           rng.integers(124, 128, (B, Hkv, cap, D // 32)).astype(np.uint8),
                           rng.integers(0, 256, (B, Hkv, cap, D // 2)).astype(np.uint8),
                           rng.integers(124, 128, (B, Hkv, cap, D // 32)).astype(np.uint8)]
        self.gamma = np.full(B, G1 - 1, np.int32) if gamma is None else np.asarray(gamma, np.int32)
        self.kv_len = (np.asarray(ctx) + self.gamma + 1).astype(np.int32)
        self.mask = None if holes is None else (rng.random((B, cap)) >= holes).astype(np.uint8)
        self.scale = float(D) ** -0.5

    def reference(self, kind, win=0, sinks=0):
        if kind == "window":
            k, v = self.k, self.v
        else:
            k, v = kv4.values(*self.cache4[:2]), kv4.values(*self.cache4[2:])
        return window.verify_attention(self.q, k, v, self.kv_len, self.gamma, self.scale, self.mask, win, sinks)

    def upload(self, kind):
        self.dq = bf16(self.q)
        self.dlen, self.dgam = dev(self.kv_len), dev(self.gamma)
        self.dmask = None if self.mask is None else dev(self.mask)
        self.dcache = [bf16(self.k), bf16(self.v)] if kind == "window" else [dev(t) for t in self.cache4]

    def workspace(self, kind, win, sinks):
        import paper_2505_07680_amd as sr

        make = sr.attention_window_workspace if kind == "window" else sr.attention_kv4_workspace
        return make(self.B, self.G1 - 1, self.Hq, self.Hkv, self.D, self.cap, win, sinks)

    def call(self, kind, win, sinks, out, ws, status=None):
        import paper_2505_07680_amd as sr

        fn = sr.specrouter_verify_attention_window if kind == "window" else sr.specrouter_verify_attention_kv4
        return fn(self.dq, *self.dcache, self.dmask, self.dlen, self.dgam, out, self.scale, win, sinks, ws, status)

    def run(self, kind, win=0, sinks=0, dtype=torch.bfloat16):
        self.upload(kind)
        out = torch.full((self.B, self.G1, self.Hq, self.D), float("nan"), dtype=dtype, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = self.workspace(kind, win, sinks)
        self.call(kind, win, sinks, out, ws, st)
        torch.cuda.synchronize()
        return out, int(st)

    def compare(self, kind, win=0, sinks=0, dtype=torch.bfloat16):
        out, st = self.run(kind, win, sinks, dtype)
        ref, size, rst = self.reference(kind, win, sinks)
        assert st == rst
        check(out, ref, size)
        return out
