// What the attention kernels over a bf16 and over a 4-bit cache share: the
// layout of a workgroup, the keys in a window's reach, and the merge of the
// streams' and the splits' softmax states.
#pragma once

#include "sr_internal.h"

namespace sr {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;  // key streams
// How far (log2) a tile's maximum exceeds a row's softmax reference before that
// is raised.
constexpr float kLazy = 8.f;
// Arrival counters sit one per 128-byte line: the splits of different
// (sequence, kv head, query chunk) jobs then never contend for one line.
constexpr int kCounterStride = 32;
// Byte offset past the end of any K/V slab (slabs are below 2^31 bytes): a
// buffer load there returns zero without touching memory.
constexpr uint32_t kOutOfRange = 0x7ffffff0u;
// Cache-policy operand of the K/V loads when one workgroup is the only
// reader of its K/V tiles (a single query chunk): non-temporal. With several
// query chunks the others re-read the same tiles, which then should stay in
// the caches (plain loads).
constexpr int kStreamLoad = 2;

// Threads, ring depth and LDS buffers per slot of a workgroup with QG query
// groups: with two groups each wave fetches half of a tile, so a four-deep
// ring of half tiles holds the registers of a two-deep ring of whole ones.
template <int QG>
struct Shape {
  static constexpr int kThreads = 64 * kWaves * QG;
  static constexpr int kRing = QG == 1 ? 2 : 4;
  static constexpr int kBufs = QG == 1 ? 1 : 2;
};

// LDS of the merge of the four stream states of each query group: the columns
// are reduced in kPasses passes so that a group's four fp32 slices fit in kMost
// bytes (72 KB: two four-wave workgroups per CU, or one of eight, fit in its 160
// KB).
constexpr int kMergeMost = 73728;
template <int D, int NQ, int QG, int kMost = kMergeMost>
struct MergeLds {
  static constexpr int MQ = 16 * NQ;
  static constexpr int kPasses = (kWaves * MQ * D * 4 <= kMost) ? 1 : (kWaves * MQ * D * 2 <= kMost) ? 2 : 4;
  static constexpr int kDp = D / kPasses;                 // columns per pass
  static constexpr int kRowStride = kDp + 4;              // floats; padded against bank conflicts
  static constexpr int kSlot = MQ * kRowStride;           // floats per wave slice
  static constexpr int kMl = QG * kWaves * kSlot * 4;     // byte offset of the (m, l) exchange
  static constexpr int kComb = kMl + QG * (kWaves + 1) * 2 * MQ * 4;
};

// 16-byte device-coherent (sc1) buffer access to the split partials; the
// descriptor's range check turns an out-of-range offset into a dropped store
// or a zero load.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t partial_rsrc(const float* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, (int)bytes, 0x00020000);
}
constexpr int kDeviceCoherent = 16;  // cache-policy operand: sc1

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __bf16 a = (__bf16)lo;
  const __bf16 b = (__bf16)hi;
  return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
}

// (the same in one instruction)
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{lo, hi}, bf16x2));
}

// A branch that is seldom taken: its code goes out of the way (a taken branch
// costs a wave about 45 cycles).
__device__ __forceinline__ bool rare(bool x) { return __builtin_expect(x, 0); }

// Order LDS accesses of one wave around a point (compiler barrier; the LDS
// unit serves one wave's requests in order).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The keys that a sequence's new rows can see, in tiles of TILE keys: with a
// window (and sinks), the tiles of the first `sinks` keys and those from the
// first key that row 0 sees on; without, all of them. Tile t of `tiles` starts at
// key start(t).
template <int TILE>
struct Reach {
  int first_key;   // row 0 sees no key before this one, but for the sinks
  int sink_tiles;  // tiles t below this start at t TILE,
  int skipped;     // the others this many tiles further on
  int tiles;
  // causal0: the position of new row 0; L: the cache's length
  __device__ __forceinline__ Reach(int causal0, int L, int window, int sinks) {
    first_key = max(causal0 - window + 1, 0);
    const int w0 = first_key / TILE;
    sink_tiles = min(sinks / TILE + (sinks % TILE != 0 ? 1 : 0), w0);
    skipped = w0 - sink_tiles;
    tiles = (L + TILE - 1) / TILE - skipped;
  }
  __device__ __forceinline__ int start(int t) const { return (t < sink_tiles ? t : t + skipped) * TILE; }
};
// The same for the host: the most tiles that any sequence's rows reach, in keys.
inline int reach_cap(int tile, int gamma_max, int L_cap, int window, int sinks) {
  if (window <= 0) return L_cap;
  const long win = ((long)window + gamma_max + 2 * tile - 2) / tile;  // (the first tile may hold one key)
  const long keys = (win + ((long)sinks + tile - 1) / tile) * tile;
  return keys < L_cap ? (int)keys : L_cap;
}

// The rows and the split that a workgroup works on. Row r of a (sequence, kv
// head) is query head r % G of the kv head's G at new row r / G.
struct JobRows {
  int row0, row_end;  // the query chunk's rows
  int Mb;             // live rows of the sequence: G (gamma_b + 1)
  int R;              // rows of a record block: G (gamma_max + 1)
  int split, ns, n_splits;  // this split, the sequence's splits that hold keys, splits of the launch
  int job;            // index of the arrival counter
  int pairs;          // (sequence, kv head) pairs of the launch
  size_t pair;        // this one
};

// Merge the streams of a workgroup and the splits of a job: o, m_run and l_run
// are the wave's unnormalised output, softmax reference (log2 units) and sum
// for its group's rows; store(r, col, x) writes four columns of an output row.
// A row whose sum is 0 (no visible key) is 0; so is one whose sum is NaN unless
// NANS, where that row is NaN (the call without a window keeps what it did).
template <class LL, int D, int NQ, int QG, int kLdsBytes, bool NANS, class Store>
__device__ __forceinline__ void merge_and_store(unsigned char* lds, const floatx4 (&o)[D / 16][NQ],
                                                const float (&m_run)[NQ], const float (&l_run)[NQ],
                                                const JobRows& J, float* part_o, float* part_ml,
                                                uint32_t* counters, const Store& store) {
  constexpr int MQ = 16 * NQ;
  constexpr int DB = D / 16;
  constexpr int kT = Shape<QG>::kThreads;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = wave_id();
  const int ws = w % kWaves;  // key stream
  const int h = w / kWaves;   // query group
  const int row0 = J.row0, row_end = J.row_end, Mb = J.Mb, R = J.R;
  const int split = J.split, ns = J.ns, n_splits = J.n_splits;
  const size_t pair = J.pair;
  const int rbase = row0 + h * MQ;
  const int l16 = lane & 15;
  const int lg = lane >> 4;

  // ---- merge the four stream states of each query group (every wave and lane takes part)
  const int tg = tid - h * 64 * kWaves;                               // thread index in the group
  float* slots = (float*)lds + h * kWaves * LL::kSlot;                  // [kWaves][MQ][kRowStride]
  float* mlx = (float*)(lds + LL::kMl) + h * (kWaves + 1) * 2 * MQ;     // [kWaves][2][MQ]: each stream's (m, l)
  float* mlf = mlx + kWaves * 2 * MQ;                                   // [2][MQ]: merged (M, L)
  if (lg == 0) {
#pragma unroll
    for (int qg = 0; qg < NQ; ++qg) {
      mlx[(ws * 2) * MQ + qg * 16 + l16] = m_run[qg];
      mlx[(ws * 2 + 1) * MQ + qg * 16 + l16] = l_run[qg];
    }
  }
  __syncthreads();
  float cw[NQ];  // this stream's weight exp2(m_w - M) per row block
#pragma unroll
  for (int qg = 0; qg < NQ; ++qg) {
    const int rl = qg * 16 + l16;
    float M = kNegInf;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) M = fmaxf(M, mlx[(v * 2) * MQ + rl]);
    float Lsum = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float c = M == kNegInf ? 0.f : exp2f(mlx[(v * 2) * MQ + rl] - M);
      Lsum += c * mlx[(v * 2 + 1) * MQ + rl];
    }
    cw[qg] = M == kNegInf ? 0.f : exp2f(m_run[qg] - M);
    if (ws == 0 && lg == 0) {
      mlf[rl] = M;
      mlf[MQ + rl] = Lsum;
    }
  }

  // With a single split holding keys the result is final here, otherwise it
  // is published as the split's partial.
  const int n_rec = (int)((size_t)n_splits * J.pairs) * R;  // records in the partial arrays
  const __amdgpu_buffer_rsrc_t rs_o = partial_rsrc(part_o, (uint32_t)((size_t)n_rec * D * 4));
  const __amdgpu_buffer_rsrc_t rs_ml = partial_rsrc(part_ml, (uint32_t)((size_t)n_rec * 8));
  constexpr int kItemsP = (MQ * (LL::kDp / 4) + 64 * kWaves - 1) / (64 * kWaves);
#pragma unroll
  for (int pass = 0; pass < LL::kPasses; ++pass) {
    __syncthreads();  // (m, l) exchange read / previous pass's slices consumed
#pragma unroll
    for (int qg = 0; qg < NQ; ++qg) {
      const int rl = qg * 16 + l16;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int col = db * 16 + lg * 4 - pass * LL::kDp;
        if (col >= 0 && col < LL::kDp) *(floatx4*)(slots + (ws * MQ + rl) * LL::kRowStride + col) = o[db][qg] * cw[qg];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItemsP; ++k) {
      const int idx = tg + k * 64 * kWaves;
      if (idx >= MQ * (LL::kDp / 4)) continue;
      const int rl = idx / (LL::kDp / 4);
      const int c4 = idx % (LL::kDp / 4);
      const int r = rbase + rl;
      if (r >= row_end) continue;
      floatx4 sum = *(const floatx4*)(slots + rl * LL::kRowStride + c4 * 4);
#pragma unroll
      for (int v = 1; v < kWaves; ++v) sum += *(const floatx4*)(slots + (v * MQ + rl) * LL::kRowStride + c4 * 4);
      const int col = pass * LL::kDp + c4 * 4;
      if (ns == 1) {
        const float Lr = mlf[MQ + rl];
        store(r, col, (r < Mb && (NANS ? Lr != 0.f : Lr > 0.f)) ? sum * (1.f / Lr) : floatx4{0.f, 0.f, 0.f, 0.f});
      } else if (r < Mb) {
        const uint32_t rec = (uint32_t)((pair * n_splits + split) * R + r);
        __builtin_amdgcn_raw_buffer_store_b128(sum, rs_o, (rec * D + col) * 4, 0, kDeviceCoherent);
        if (pass == 0 && c4 == 0)
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, floatx2{mlf[rl], mlf[MQ + rl]}), rs_ml, rec * 8, 0, kDeviceCoherent);
      }
    }
  }
  if (ns == 1) return;

  // ---- arrive: the last split of this job to finish merges all partials
  stores_done();
  __syncthreads();
  __shared__ uint32_t last_flag;
  if (tid == 0) {
    uint32_t* cnt = counters + (size_t)J.job * kCounterStride;
    const uint32_t before = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == (uint32_t)(ns - 1);
    if (last) st_dev(cnt, 0u);  // every split of this job has arrived: reset for the next call
    last_flag = last ? 1u : 0u;
  }
  __syncthreads();
  if (last_flag == 0u) return;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);

  // Merge: out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the splits, M
  // their largest reference. Bound by the latency of the partials' device-coherent
  // loads (one to two us a round trip, from another XCD's write), so as many as
  // registers hold are in flight: first the first kGroup splits' outputs and
  // every (m, l), then the remaining groups, with the weights from the (m, l) in
  // LDS. (A running maximum over groups of four splits, their (m, l) beside the
  // outputs, took 0.33 us per split at 24 rows of 128 columns; this takes
  // 0.2.) Each thread owns kItems (row, 4 columns) items.
  constexpr int kItems = (QG * MQ * (D / 4) + kT - 1) / kT;
  // (registers: 32 to 96, fewer than the key loop's)
  constexpr int kGroup = kItems >= 3 ? 4 : 8;
  constexpr int kMlBlock = 64;  // splits whose references sit in LDS at once
  constexpr int kRows = QG * MQ;
  static_assert((2 + kMlBlock) * kRows * 4 <= kLdsBytes, "the merge's exchange fits");
  const int n_rows = row_end - row0;
  const int n_items = n_rows * (D / 4);
  float* mM = (float*)lds;           // [kRows] M
  float* mD = mM + kRows;            // [kRows] denominators
  float* mS = mD + kRows;            // [kMlBlock][kRows] m_s
  const uint32_t rec0 = (uint32_t)(pair * n_splits * R);
  const __amdgpu_buffer_rsrc_t rs_none = partial_rsrc(part_o, 0);
  auto live_row = [&](int row) __attribute__((always_inline)) { return min(row0 + row, Mb - 1); };  // (rows past Mb hold no partial; their result is discarded)
  // (past the splits: an empty resource, zeros without traffic)
  auto sp_rsrc = [&](int sp, const __amdgpu_buffer_rsrc_t& rs) __attribute__((always_inline)) { return sp < ns ? rs : rs_none; };
  auto fetch_o = [&](int sp0, floatx4 (&o2)[kGroup][kItems]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int idx = min(tid + k * kT, n_items - 1);
        const uint32_t rec = rec0 + (uint32_t)((sp0 + j) * R + live_row(idx / (D / 4)));
        o2[j][k] = __builtin_amdgcn_raw_buffer_load_b128(sp_rsrc(sp0 + j, rs_o), (rec * D + (idx % (D / 4)) * 4) * 4, 0, kDeviceCoherent);
      }
  };
  auto write_item = [&](int k, const floatx4& sum, float den) __attribute__((always_inline)) {
    const int idx = tid + k * kT;
    if (idx >= n_items) return;
    const int r = row0 + idx / (D / 4);
    const bool live = r < Mb && (NANS ? den != 0.f : den > 0.f);
    store(r, (idx % (D / 4)) * 4, live ? sum * (1.f / den) : floatx4{0.f, 0.f, 0.f, 0.f});
  };
  floatx4 o2[kGroup][kItems];
  fetch_o(0, o2);
  __builtin_amdgcn_sched_barrier(0);
  constexpr int kFew = 4;
  if (kItems <= 4 && ns <= kFew) {  // one round trip: every thread takes its rows' (m, l) itself (0.4 us less than through LDS)
#pragma unroll
    for (int k = 0; k < (kItems <= 4 ? kItems : 0); ++k) {
      const int row = live_row(min(tid + k * kT, n_items - 1) / (D / 4));
      floatx2 x[kFew];
#pragma unroll
      for (int j = 0; j < kFew; ++j)
        x[j] = __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(sp_rsrc(j, rs_ml), (rec0 + (uint32_t)(j * R + row)) * 8, 0, kDeviceCoherent));
      float M = kNegInf, den = 0.f;
#pragma unroll
      for (int j = 0; j < kFew; ++j) M = j < ns ? fmaxf(M, x[j].x) : M;
      floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kFew; ++j) {
        const float wgt = j < ns && x[j].x != kNegInf ? exp2_hw(x[j].x - M) : 0.f;
        den += x[j].y * wgt;
        sum += o2[j][k] * wgt;
      }
      write_item(k, sum, den);
    }
    return;
  }
  // (m, l) of every split: four threads per row take the splits in turn. A split
  // whose scores were all NaN has reference -inf and sum NaN, which NANS passes on.
  constexpr float kNone = NANS ? 1.f : 0.f;
  for (int row = tid / 4; row < n_rows; row += kT / 4) {
    constexpr int kMl = 8;
    float M = kNegInf, den = 0.f;
    const uint32_t rec = rec0 + (uint32_t)live_row(row);
    for (int sp0 = tid % 4; sp0 < ns; sp0 += 4 * kMl) {
      floatx2 x[kMl];
#pragma unroll
      for (int j = 0; j < kMl; ++j)
        x[j] = __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(
                                               rs_ml, sp0 + 4 * j < ns ? (rec + (uint32_t)((sp0 + 4 * j) * R)) * 8 : kOutOfRange, 0, kDeviceCoherent));
      float Mn = M;
#pragma unroll
      for (int j = 0; j < kMl; ++j) Mn = sp0 + 4 * j < ns ? fmaxf(Mn, x[j].x) : Mn;
      den = Mn == kNegInf ? den * kNone : den * exp2_hw(M - Mn);
#pragma unroll
      for (int j = 0; j < kMl; ++j) {
        const int sp = sp0 + 4 * j;
        if (sp < ns) {
          if (NANS || Mn != kNegInf) den += x[j].y * (Mn == kNegInf ? 1.f : exp2_hw(x[j].x - Mn));
          if (sp < kMlBlock) mS[sp * kRows + row] = x[j].x;
        }
      }
      M = Mn;
    }
    // the row's four threads (a quad): (M, den) over all splits
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      const float Mo = d == 1 ? perm_f32<dpp::kXor1>(M) : perm_f32<dpp::kXor2>(M);
      const float Do = d == 1 ? perm_f32<dpp::kXor1>(den) : perm_f32<dpp::kXor2>(den);
      const float Mn = fmaxf(M, Mo);
      // (the fused operand is written out, so that every kernel rounds alike)
      den = Mn == kNegInf ? (den + Do) * kNone : fmaf(den, exp2_hw(M - Mn), Do * exp2_hw(Mo - Mn));
      M = Mn;
    }
    if (tid % 4 == 0) {
      mM[row] = M;
      mD[row] = den;
    }
  }
  floatx4 acc[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) acc[k] = floatx4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  for (int b0 = 0; b0 < ns; b0 += kMlBlock) {
    if (b0 > 0) {  // the next block's references
      __syncthreads();
      for (int i = tid; i < min(ns - b0, kMlBlock) * n_rows; i += kT) {
        const int sp = i / n_rows, row = i % n_rows;
        mS[sp * kRows + row] = __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(
                                                             rs_ml, (rec0 + (uint32_t)((b0 + sp) * R + live_row(row))) * 8, 0, kDeviceCoherent)).x;
      }
      __syncthreads();
    }
    const int b1 = min(ns, b0 + kMlBlock);
    for (int sp0 = b0; sp0 < b1; sp0 += kGroup) {
      if (sp0 > 0) fetch_o(sp0, o2);
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int row = min(tid + k * kT, n_items - 1) / (D / 4);
        const float M = mM[row];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
          const float m = mS[(sp0 + j < b1 ? sp0 + j - b0 : 0) * kRows + row];
          const float wgt = sp0 + j < b1 && m != kNegInf ? exp2_hw(m - M) : 0.f;
          acc[k] += o2[j][k] * wgt;
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kItems; ++k) write_item(k, acc[k], mD[min(tid + k * kT, n_items - 1) / (D / 4)]);
}

}  // namespace
}  // namespace sr
