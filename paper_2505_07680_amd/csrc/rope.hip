// The new queries and keys of a step, or of a prompt, before the cache is
// written: every head divided by its root mean square and weighted, then
// rotated by its position.
//
//   y = x rsqrt(mean(x^2) + eps) w        (or y = x, without weights)
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
//
// over the pairs (a, b) of the rotated part, t the pair's angle at the row's
// position, from a table. Everything in 32 bits, rounded to bf16 once.
//
// A head takes D/8 lanes of eight values each (one 16-byte load and store), so a
// wave holds 4 heads of 128 or 8 of 64 at a time, all of one token: the angles are
// loaded once and stay in registers for the wave's few steps, whose loads are all
// in flight before the first is used. With pairs half a rotation apart the
// partner's values come from the lane that holds them, by way of the LDS crossbar.
//
// Bound by HBM for prompts: 4 of 8100 rows, 72 heads of 128, 190 us, 6.3 TB/s read
// and written (a large device copy reaches 4.9). 256 sequences' steps (30 MB)
// take 9.8 us, 3.0 TB/s: the launch, the cold caches and one wave's chain of
// position, loads, angles and store. One token takes 2.5 us, the launch.

#include "caching.h"

namespace sr {
namespace {

constexpr int kRopeThreads = 256;
// Steps of a wave. While the data comes from or stays in a cache, twice the waves
// hide more than a longer wave's loads and the reuse of its angles save (40 heads
// of 128, us with two and with four steps: one token 2.4 and 2.7, 192 tokens 3.4
// and 4.2, 1443 tokens 9.7 and 11.1, 4096 tokens 20.7 and 21.5);
// streamed from HBM it is the other way round (333 MB 64 and 58, 1.2 GB 195 and 190).
constexpr int head_steps(int caching) { return caching == kPass ? 4 : 2; }
// A mean of squares from here to 32 bits' largest has all its bits: a square that counts, from
// 2^-24 of the largest on, is not below 2^-126.
constexpr float kLeastMean = 0x1p-96f;

__device__ __forceinline__ float lane_f32(float x, int src_lane) {
  return __int_as_float(__builtin_amdgcn_ds_bpermute(src_lane * 4, __float_as_int(x)));
}

__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  const __bf16 a = (__bf16)lo;
  const __bf16 b = (__bf16)hi;
  return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
}

// Eight weights from element c8 on, widened to 32 bits.
__device__ __forceinline__ void load_weights(const void* w, bool f32, int c8, float (&out)[8]) {
  if (f32) {
    const float4* p = (const float4*)((const float*)w + c8);
    const float4 a = p[0], b = p[1];
    out[0] = a.x, out[1] = a.y, out[2] = a.z, out[3] = a.w;
    out[4] = b.x, out[5] = b.y, out[6] = b.z, out[7] = b.w;
  } else {
    const u32x4 x = *(const u32x4*)((const uint16_t*)w + c8);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      out[2 * e] = bf16_lo(x[e]);
      out[2 * e + 1] = bf16_hi(x[e]);
    }
  }
}

template <int D, bool ADJACENT, int CACHING>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_kernel(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                    const void* __restrict__ qw, const void* __restrict__ kw, bool w_f32, float eps,
                    const float* __restrict__ table, int max_positions, int rot,
                    const int32_t* __restrict__ position, const int32_t* __restrict__ gamma, uint16_t* q_out,
                    uint16_t* k_out, int gmax, int Hq, int Hkv, int parts, uint32_t n_items, int32_t* __restrict__ status) {
  constexpr int kLanes = D / 8;        // lanes per head
  constexpr int kHeads = 64 / kLanes;  // heads per step of a wave
  constexpr int kHeadSteps = head_steps(CACHING);
  // item: (token, part of its heads)
  const uint32_t item = blockIdx.x * (kRopeThreads / 64) + (uint32_t)wave_id();
  if (item >= n_items) return;
  const int64_t token = item / (uint32_t)parts;
  const int part = (int)(item % (uint32_t)parts);
  const int b = (int)((uint32_t)token / (uint32_t)(gmax + 1));
  const int i = (int)((uint32_t)token % (uint32_t)(gmax + 1));
  const int gam = gamma[b], pos0 = position[b];
  const bool g_ok = gam >= 0 && gam <= gmax;
  const bool ok = g_ok && pos0 >= 0 && pos0 < max_positions - gam;
  const int lane = threadIdx.x & 63;
  if (!ok) {
    if (i == 0 && part == 0 && lane == 0 && status) atomicOr(status, g_ok ? SR_ST_POSITION : SR_ST_GAMMA);
    return;
  }
  if (i > gam) return;

  const int c = lane % kLanes;  // elements 8 c .. 8 c + 7 of the head
  const int H = Hq + Hkv;
  const int h0 = part * (kHeads * kHeadSteps) + lane / kLanes;
  u32x4 x[kHeadSteps];
#pragma unroll
  for (int s = 0; s < kHeadSteps; ++s) {
    const int h = min(h0 + s * kHeads, H - 1);
    const uint16_t* src = h < Hq ? q + token * q_stride + (int64_t)h * D : k + token * k_stride + (int64_t)(h - Hq) * D;
    x[s] = load_once<CACHING>(src + c * 8);
  }
  float wq[8], wk[8];
  if (qw) load_weights(qw, w_f32, c * 8, wq);
  if (kw) load_weights(kw, w_f32, c * 8, wk);
  const bool turns = c * 8 < rot;
  // angles of this lane's elements: cosines, then sines, rot/2 of each per position
  const float* row = table + (int64_t)(pos0 + i) * rot;
  constexpr int kAngles = ADJACENT ? 4 : 8;
  const int half = rot / 16;  // chunks of eight in half of the rotated part
  const int a0 = !turns ? 0 : ADJACENT ? c * 4 : (c < half ? c : c - half) * 8;
  float cs[kAngles], sn[kAngles];
#pragma unroll
  for (int e = 0; e < kAngles; e += 4) {
    const float4 u = *(const float4*)(row + a0 + e), v = *(const float4*)(row + rot / 2 + a0 + e);
    cs[e] = u.x, cs[e + 1] = u.y, cs[e + 2] = u.z, cs[e + 3] = u.w;
    sn[e] = v.x, sn[e + 1] = v.y, sn[e + 2] = v.z, sn[e + 3] = v.w;
  }
  const int partner = lane - c + (!turns ? c : c < half ? c + half : c - half);
  const float sign = c < half ? -1.f : 1.f;
#pragma unroll
  for (int s = 0; s < kHeadSteps; ++s) {
    const int h = h0 + s * kHeads;
    const bool is_q = h < Hq;
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[2 * e] = bf16_lo(x[s][e]);
      y[2 * e + 1] = bf16_hi(x[s][e]);
    }
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
    ss += perm_f32<dpp::kXor1>(ss);
    ss += perm_f32<dpp::kXor2>(ss);
    ss += perm_f32<dpp::kHalfMirror>(ss);
    if constexpr (kLanes == 16) ss += perm_f32<dpp::kMirror>(ss);
    float ms = ss * (1.f / D) + eps;
    // Squares beyond 32 bits' range, or so small that they lose bits: the head again, divided
    // by the power of two above its largest magnitude (and above sqrt(eps)), which is exact.
    const bool scaled = __float_as_uint(ms) - __float_as_uint(kLeastMean) >= 0x7f800000u - __float_as_uint(kLeastMean);
    if (__builtin_expect(__ballot(scaled) != 0ull, 0)) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
      top = max(top, perm_u32<dpp::kXor1>(top));
      top = max(top, perm_u32<dpp::kXor2>(top));
      top = max(top, perm_u32<dpp::kHalfMirror>(top));
      if constexpr (kLanes == 16) top = max(top, perm_u32<dpp::kMirror>(top));
      // (an infinity or a NaN, and a head without a norm, stay as they are)
      const bool at_all = scaled && top < 0x7f800000u && (is_q ? qw != nullptr : kw != nullptr);
      const int of_eps = eps > 0.f ? (__builtin_amdgcn_frexp_expf(eps) + 1) / 2 : -1000;
      const int power = at_all ? max(__builtin_amdgcn_frexp_expf(__uint_as_float(top)), of_eps) : 0;
      ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = ldexpf(y[e], -power);
        ss = fmaf(y[e], y[e], ss);
      }
      ss += perm_f32<dpp::kXor1>(ss);
      ss += perm_f32<dpp::kXor2>(ss);
      ss += perm_f32<dpp::kHalfMirror>(ss);
      if constexpr (kLanes == 16) ss += perm_f32<dpp::kMirror>(ss);
      ms = ss * (1.f / D) + ldexpf(eps, -2 * power);
    }
    const float rs = rsqrtf(ms);
    if (is_q ? qw != nullptr : kw != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= rs * (is_q ? wq[e] : wk[e]);
    }
    float z[8];
    if constexpr (ADJACENT) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = y[2 * e], v = y[2 * e + 1];
        z[2 * e] = turns ? u * cs[e] - v * sn[e] : u;
        z[2 * e + 1] = turns ? v * cs[e] + u * sn[e] : v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float o = lane_f32(y[e], partner);  // (every lane of the wave takes part)
        z[e] = turns ? y[e] * cs[e] + sign * o * sn[e] : y[e];
      }
    }
    if (h < H) {
      uint16_t* dst = is_q ? q_out + (token * Hq + h) * D : k_out + (token * Hkv + (h - Hq)) * D;
      store_once<CACHING>(dst + c * 8, u32x4{to_bf16x2(z[0], z[1]), to_bf16x2(z[2], z[3]), to_bf16x2(z[4], z[5]),
                                             to_bf16x2(z[6], z[7])});
    }
  }
}

template <int CACHING>
auto rope_kernel(int D, bool adjacent) {
  return D == 64 ? (adjacent ? qk_norm_rope_kernel<64, true, CACHING> : qk_norm_rope_kernel<64, false, CACHING>)
                 : (adjacent ? qk_norm_rope_kernel<128, true, CACHING> : qk_norm_rope_kernel<128, false, CACHING>);
}

}  // namespace

int launch_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* q_weight,
                        const void* k_weight, bool w_f32, float eps, const float* table, int max_positions, int rot,
                        bool adjacent, const int32_t* position, const int32_t* gamma, void* q_out, void* k_out, int B,
                        int gamma_max, int Hq, int Hkv, int D, int32_t* status, hipStream_t stream) {
  // Queries and keys from the same rows, one of them in place: the other first, in a launch of its own.
  if (q == k && (q_out == q || k_out == k)) {
    const auto queries = [&] {
      return launch_qk_norm_rope(q, q_stride, nullptr, 0, q_weight, nullptr, w_f32, eps, table, max_positions, rot,
                                 adjacent, position, gamma, q_out, k_out, B, gamma_max, Hq, 0, D, status, stream);
    };
    const auto keys = [&] {
      return launch_qk_norm_rope(nullptr, 0, k, k_stride, nullptr, k_weight, w_f32, eps, table, max_positions, rot,
                                 adjacent, position, gamma, q_out, k_out, B, gamma_max, 0, Hkv, D, status, stream);
    };
    const int rc = q_out == q ? keys() : queries();
    return rc != SR_OK ? rc : q_out == q ? queries() : keys();
  }
  const Caching caching = caching_of((long)B * (gamma_max + 1) * (Hq + Hkv) * D * 4);
  const int per_wave = 64 / (D / 8) * head_steps(caching);
  const int parts = (Hq + Hkv + per_wave - 1) / per_wave;
  const long n_items = (long)B * (gamma_max + 1) * parts;
  const long blocks = (n_items + kRopeThreads / 64 - 1) / (kRopeThreads / 64);
  if (blocks * kRopeThreads >= 1l << 32) return SR_EINVAL;  // (a launch's threads are counted in 32 bits)
  const auto kernel = caching == kPass ? rope_kernel<kPass>(D, adjacent)
                                       : caching == kReadOnce ? rope_kernel<kReadOnce>(D, adjacent)
                                                              : rope_kernel<kKeep>(D, adjacent);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRopeThreads), 0, stream, (const uint16_t*)q, q_stride,
                     (const uint16_t*)k, k_stride, q_weight, k_weight, w_f32, eps, table, max_positions, rot, position,
                     gamma, (uint16_t*)q_out, (uint16_t*)k_out, gamma_max, Hq, Hkv, parts, (uint32_t)n_items, status);
  return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
}

}  // namespace sr
