// A K/V cache held in 4 bits: the rows written to it.
//
// A row's 32 elements take one power of two 2^(p - 127), the least (p from 1 to
// 252) of which the largest element is at most 7, and each element the nearest
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it with a sign (e2m1; of two equally near
// the one with the even code). Elements between 6 and 7 powers become 6: off by at
// most the half step that those between 4 and 6 are off by. An element over its
// power is exact (both bf16), so the codes are a function of the row alone. A
// group that holds an infinity or a NaN gets p = 255, which reads as NaN.
//
// Four lanes take a group of 32 (a 16-byte load of eight bf16 each; the group's
// largest magnitude is an integer maximum over the four); the conversion is the
// hardware's (v_cvt_scalef32_pk_fp4_bf16 divides by the power of two and rounds to
// nearest even). A wave takes consecutive positions of one head, so that its
// stores are one run of the head's slab.
//
// Prompts are bound by HBM and their many short runs (8 KB to 2 KB apart in what is
// read; powers of 4 bytes a row at D = 128, 2 at 64, 16 to a wave's rows): 8 of 2048 to
// 4095 rows, 8 heads of 128, with the values that attention will see, 228 MB, 40 us in
// the rows' kernel (5.7 TB/s) and 4 in the lengths'. A step's rows are bound by latency:
// 5.2 us for 256 sequences (13 MB), of which the launch is about half.

#include "caching.h"

namespace sr {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight elements of a row (four lanes hold a group of 32): their codes, and the group's power.
struct Rounded {
  uint32_t codes;
  uint32_t power;
};
__device__ __forceinline__ Rounded round_to_4_bits(const u32x4& x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7fffu, (x[e] >> 16) & 0x7fffu));
  top = max(top, perm_u32<dpp::kXor1>(top));
  top = max(top, perm_u32<dpp::kXor2>(top));
  const bool odd = top >= 0x7f80u;  // an infinity or a NaN among the 32
  // the exponent of top, one more where its mantissa is above 1.75, less 2
  const uint32_t p = (uint32_t)min(max((int)((top + 0x1fu) >> 7) - 2, 1), 252);
  const float scale = __uint_as_float(p << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[2]), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[3]), scale, 3);
  return {odd ? 0u : c, odd ? 255u : p};
}

// The bf16 values that the codes stand for (NaN throughout a group with p = 255).
__device__ __forceinline__ u32x4 values_of(const Rounded& r) {
  const float scale = __uint_as_float(r.power << 23);
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, scale, 0));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, scale, 1));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, scale, 2));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, scale, 3));
  return r.power == 255u ? u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u} : v;
}

struct Append4 {
  const uint16_t *k_new, *v_new;
  int64_t k_stride, v_stride;  // elements from a token to the next
  const int32_t* gamma;
  uint8_t *k_codes, *k_powers, *v_codes, *v_powers;
  uint8_t* mask;
  int32_t* kv_len;
  const int32_t* shared_len;
  uint16_t *k_seen, *v_seen;
  int gmax, Hkv, L_cap;
  int32_t* status;
};

// The cursor and the rows of sequence b: n = 0 for bad data (its SR_ST_* bit in bad).
struct Span {
  int cur, n;
  int32_t bad;
};
__device__ __forceinline__ Span span_of(const Append4& a, int b) {
  const int g = a.gamma[b], L = a.kv_len[b];
  const int cur = a.shared_len ? *a.shared_len : L;
  int32_t bad = 0;
  if (g < 0 || g > a.gmax) bad = SR_ST_GAMMA;
  else if (L < 0 || L > a.L_cap || cur < 0 || cur > a.L_cap - (g + 1)) bad = SR_ST_KVLEN;
  return {cur, bad ? 0 : g + 1, bad};
}

// Rows [first, first + kU * step) in steps of the sequence's n Hkv rows, head by
// head; a lane takes its eight elements of every one (kU loads of K and V in flight).
template <int D, int kU, int CACHING>
__device__ __forceinline__ void append_rows(const Append4& a, int b, int cur, int n, int first, int step, int total) {
  constexpr int kLanes = D / 8;
  const int c = (int)(threadIdx.x % kLanes);
  u32x4 kr[kU], vr[kU];
  int h[kU], i[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const int row = min(first + u * step, total - 1);
    h[u] = row / n;
    i[u] = row - h[u] * n;
    const int64_t token = (int64_t)b * (a.gmax + 1) + i[u];
    kr[u] = load_once<CACHING>(a.k_new + token * a.k_stride + (int64_t)h[u] * D + c * 8);
    vr[u] = load_once<CACHING>(a.v_new + token * a.v_stride + (int64_t)h[u] * D + c * 8);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const Rounded k4 = round_to_4_bits(kr[u]), v4 = round_to_4_bits(vr[u]);
    if (first + u * step < total) {
      const int64_t slot = ((int64_t)b * a.Hkv + h[u]) * a.L_cap + cur + i[u];
      ((uint32_t*)a.k_codes)[slot * kLanes + c] = k4.codes;
      ((uint32_t*)a.v_codes)[slot * kLanes + c] = v4.codes;
      if ((c & 3) == 0) {
        a.k_powers[slot * (D / 32) + c / 4] = (uint8_t)k4.power;
        a.v_powers[slot * (D / 32) + c / 4] = (uint8_t)v4.power;
      }
      const int64_t seen = ((((int64_t)b * (a.gmax + 1) + i[u]) * a.Hkv + h[u]) * D) + c * 8;
      if (a.k_seen) store_once<CACHING>(a.k_seen + seen, values_of(k4));
      if (a.v_seen) store_once<CACHING>(a.v_seen + seen, values_of(v4));
    }
  }
}

// Few rows: one workgroup per sequence, which reads the cursor once and
// then is the only writer of the length.
constexpr int kStepThreads = 1024;
template <int D>
__global__ void __launch_bounds__(kStepThreads)
kv4_append_step_kernel(Append4 a) {
  constexpr int kRows = kStepThreads / (D / 8);
  const int b = blockIdx.x;
  const Span s = span_of(a, b);
  __syncthreads();  // every thread has read the length
  if (s.n == 0) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status, s.bad);
    return;
  }
  const int total = s.n * a.Hkv;
  for (int first = (int)threadIdx.x / (D / 8); first < total; first += kRows)
    append_rows<D, 1, kKeep>(a, b, s.cur, s.n, first, kRows, total);
  if (a.mask)
    for (int i = threadIdx.x; i < s.n; i += kStepThreads) a.mask[(int64_t)b * a.L_cap + s.cur + i] = 1;
  if (threadIdx.x == 0) a.kv_len[b] = s.cur + s.n;
}

// More: workgroups over blocks of rows; the lengths and the mask follow in a
// kernel of their own, when every row's workgroup has read the cursor.
constexpr int kPromptThreads = 256;
constexpr int kPromptUnroll = 4;
template <int D>
constexpr int prompt_rows() { return kPromptThreads / (D / 8) * kPromptUnroll; }
template <int D, int CACHING>
__global__ void __launch_bounds__(kPromptThreads)
kv4_append_prompt_kernel(Append4 a, int blocks_per_seq) {
  constexpr int kRows = 64 / (D / 8);  // rows of a wave at a time
  const int b = (int)(blockIdx.x / (unsigned)blocks_per_seq);
  const int blk = (int)(blockIdx.x % (unsigned)blocks_per_seq);
  const Span s = span_of(a, b);
  const int total = s.n * a.Hkv;
  const int lane = threadIdx.x & 63;
  const int first = blk * prompt_rows<D>() + wave_id() * (kRows * kPromptUnroll);
  if (first >= total) return;
  append_rows<D, kPromptUnroll, CACHING>(a, b, s.cur, s.n, first + lane / (D / 8), kRows, total);
}

constexpr int kLenThreads = 256;
__global__ void __launch_bounds__(kLenThreads)
kv4_append_length_kernel(Append4 a) {
  const int b = blockIdx.x;
  const Span s = span_of(a, b);
  __syncthreads();
  if (s.n == 0) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status, s.bad);
    return;
  }
  if (a.mask)
    for (int i = threadIdx.x; i < s.n; i += kLenThreads) a.mask[(int64_t)b * a.L_cap + s.cur + i] = 1;
  if (threadIdx.x == 0) a.kv_len[b] = s.cur + s.n;
}

template <int CACHING>
auto prompt_kernel(int D) {
  return D == 64 ? kv4_append_prompt_kernel<64, CACHING> : kv4_append_prompt_kernel<128, CACHING>;
}

}  // namespace

// Whether one workgroup appends a sequence's rows (all heads counted): up to three of
// its passes, where one launch less is worth more than more CUs, and up to eight where
// such workgroups fill more than half of the CUs in one turn. us with one workgroup
// and with blocks of rows, heads of 128, 64 rows a pass, inputs from HBM:
//   sequences   3 passes    4           6           8           16
//        16     7.5  7.6    8.6  7.8   11.2  7.9   13.7  8.1   29.0 10.3
//        64     8.9  9.3   11.8 10.0   16.4 12.5   20.3 14.0   36.7 20.0
//       128    11.6 13.2   13.8 14.1   19.1 15.5   22.8 20.5   42.4 33.7
//       160    12.2 14.3   15.0 15.1   20.3 19.8   25.3 25.1   45.9 40.6
//       224    14.4 16.0   17.7 20.1   24.4 25.7   30.7 34.2   56.6 53.6
//       256    15.3 16.1   18.8 20.2   26.4 26.6   33.7 34.4   65.2 59.9
//       320    22.2 20.7   26.8 23.8   38.6 34.3   48.9 41.2   96.7 72.9
// One sequence: 6.6 and 6.6 with 3, 21.5 and 6.7 with 16. Heads of 64, 128 rows a pass: the same
// within 10%.
bool one_workgroup_each(int B, long rows, int D, int cus) {
  const long passes = (rows * D + kStepThreads * 8 - 1) / (kStepThreads * 8);
  return passes <= 3 || (passes <= 8 && B > cus / 2 && B <= cus);
}

int launch_kv4_append(const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, const int32_t* gamma,
                      void* k_codes, void* k_powers, void* v_codes, void* v_powers, uint8_t* cache_mask,
                      int32_t* kv_len, const int32_t* shared_len, void* k_seen, void* v_seen, int B, int gamma_max,
                      int Hkv, int D, int L_cap, int32_t* status, hipStream_t stream) {
  const Append4 a{(const uint16_t*)k_new, (const uint16_t*)v_new, k_stride, v_stride, gamma,
                  (uint8_t*)k_codes, (uint8_t*)k_powers, (uint8_t*)v_codes, (uint8_t*)v_powers, cache_mask, kv_len,
                  shared_len, (uint16_t*)k_seen, (uint16_t*)v_seen, gamma_max, Hkv, L_cap, status};
  const long rows = (long)(gamma_max + 1) * Hkv;
  const int cus = device_cu_count();
  if (cus <= 0) return SR_ELAUNCH;
  if (one_workgroup_each(B, rows, D, cus)) {
    hipLaunchKernelGGL(D == 64 ? kv4_append_step_kernel<64> : kv4_append_step_kernel<128>, dim3(B), dim3(kStepThreads),
                       0, stream, a);
    return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
  }
  const int per = D == 64 ? prompt_rows<64>() : prompt_rows<128>();
  const int blocks = (int)((rows + per - 1) / per);
  if ((long)B * blocks * kPromptThreads >= 1l << 32) return SR_EINVAL;  // (a launch's threads are counted in 32 bits)
  const Caching caching = caching_of((long)B * rows * D * 4 * (k_seen || v_seen ? 2 : 1));
  const auto kernel = caching == kPass ? prompt_kernel<kPass>(D)
                                       : caching == kReadOnce ? prompt_kernel<kReadOnce>(D) : prompt_kernel<kKeep>(D);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long)B * blocks)), dim3(kPromptThreads), 0, stream, a, blocks);
  if (hipGetLastError() != hipSuccess) return SR_ELAUNCH;
  hipLaunchKernelGGL(kv4_append_length_kernel, dim3(B), dim3(kLenThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
}

}  // namespace sr
