// Verification attention for gfx950 (Section 2.2 step 2; Section 4.4, Eq. 8).
//
// Work decomposition. One workgroup handles one (sequence b, kv head g, query
// chunk, key split). All G*(gamma_b+1) query rows that read kv head g (the GQA
// group times the new positions) are processed together, so every K/V byte of
// the split is read from HBM exactly once. Four key streams: stream s owns 16
// of every 64 keys and keeps its own online-softmax state; the four states
// are merged through LDS at the end. Up to 48 query rows, a workgroup is four
// waves, one per stream, with no workgroup barrier inside the key loop. Up
// to 96 rows it is eight waves in two query groups: the two waves of a
// stream each fetch half of every K/V tile into a shared LDS slot (two tiles at
// a time, a workgroup barrier before and after their compute) and each computes
// its own group's rows over both, so a tile is still read once. When the
// cache is split, each split publishes its (max, sum, unnormalised output)
// partial and bumps a per-(b, g, query chunk) arrival counter; the last
// workgroup to arrive merges all partials in split order and writes the
// output, then resets the counter, so the workspace is left ready for the
// next call. The summation order is fixed, so results are reproducible.
// When the workgroups outnumber what the device holds at once, a small
// kernel first sorts the jobs by key count and the workgroups take them
// longest first, so that the device does not idle behind a few long
// workgroups at the end of a ragged batch.
//
// Per 16-key tile of a stream:
//   * K and V rows are fetched with coalesced 16-byte loads into a register
//     ring (two tiles deep, or four half tiles with two query groups), so
//     loads stay in flight while a tile is computed, and staged in the
//     stream's LDS slot; rows at or past kv_len are fetched
//     out of the buffer range (they read as zero, with no memory traffic) and
//     V rows under mask 0 are zeroed while staging, so whatever those rows
//     hold never reaches the output;
//   * S^T = K Q^T on MFMA (v_mfma_f32_16x16x32_bf16: 16 keys x 16 queries per
//     block, K=32 over the head dimension); each lane then holds 4 scores of
//     ONE query, so the softmax max/sum need only two cross-lane steps;
//   * the softmax reference of a row is raised to a tile's maximum only when
//     that exceeds it by more than 2^8, so the output accumulators are rarely
//     rescaled; where fewer splits than one workgroup per CU take the least time it
//     also moves within one binade with every tile (see next_ref and
//     attention_plan), which rescales them by less than 2 each time;
//   * P is rounded to bf16 in place: its accumulator layout is exactly the B
//     operand of O^T += V^T P^T (v_mfma_f32_16x16x16_bf16, K=16 over the keys;
//     with two query groups v_mfma_f32_16x16x32_bf16 over two tiles' keys); the
//     V^T operand comes from the LDS transposing read.
// Scores are kept in log2 units (scale * log2(e) folded in) and exponentiated
// with exp2.
//
// With a window (WIN) a row at position pos sees the keys above pos - window and
// the cache's first `sinks`. Only the tiles that hold such keys are taken: they
// are numbered without the gap between the sinks and row 0's first key, and
// splits and streams deal those numbers as they deal all tiles otherwise. V rows
// that no row sees are zeroed like masked ones. Its softmax takes a row's sum across
// lanes at the end and its maximum only when the reference grows (or follows the
// tiles, where the call without a window would have it follow), masks by
// putting -infinity in the scores' place, and with one query group leaves row
// blocks without live rows out of the products too (the loop is compiled for
// each number of them): 64 sequences of 1024 positions, gamma 1 to 8, 58 -> 53 us,
// 16 of 4096 with 72 rows 75 -> 67. More than 48 rows mostly go to chunks of four waves
// instead of eight waves (see attention_plan). The kernel without a window is compiled apart
// and keeps its own arithmetic.

#pragma once

#include <type_traits>

#include "attention_common.h"

namespace sr {
namespace {

constexpr int kWaveKeys = 16;
// At most three 16-row query blocks per wave (the accumulators stay in 256
// registers at two waves per SIMD) and two query groups per workgroup: more
// than 96 rows go to further query chunks, which read the same K/V again.
constexpr int kMaxNQ = 3;
constexpr int kMaxQG = 2;
// The same where the reference follows the tiles.
constexpr float kLazyFollow = 7.f;
constexpr int kMaxSplitKeys = 8448;  // keys per split at most (about 4 MB of K/V at D = 128)

template <int D>
struct Geo {
  static constexpr int kKStride = D * 2 + 16;  // LDS bytes per staged K (and Q) row
  // LDS bytes per staged V row: four consecutive rows' 32-byte column blocks
  // fall on different banks for the transposing reads of the V^T operand
  static constexpr int kVStride = D * 2 + 32;
  static constexpr int kChunksPerRow = D / 8;  // 16-byte chunks per row
  static constexpr int kRowsPerLoad = 64 / kChunksPerRow;
  static constexpr int kLoads = kWaveKeys / kRowsPerLoad;  // 16-byte loads per lane per tensor per tile
  static constexpr int kSlotK = kWaveKeys * kKStride;
  static constexpr int kWaveBytes = kSlotK + kWaveKeys * kVStride;
};

template <int D, int NQ, int QG>
struct Lds {
  static constexpr int MQ = 16 * NQ;
  static constexpr int kStage = kWaves * Shape<QG>::kBufs * Geo<D>::kWaveBytes + QG * MQ * Geo<D>::kKStride;
  static constexpr int kComb = MergeLds<D, NQ, QG>::kComb;
  static constexpr int kBytes = kStage > kComb ? kStage : kComb;
};

template <int D, int QG>
struct Stage {  // one wave's part of a 16-key tile in flight
  u32x4 k[Geo<D>::kLoads / QG], v[Geo<D>::kLoads / QG];
  uint32_t mbyte;  // validity byte of key (lane mod 16), evaluated when consumed
};

// A row's softmax reference (log2 units) for a tile whose largest score is mt,
// m_run being the one before; grow: mt is far above that (or the row's first).
// Lazy: the reference stays unless it grows, to mt. Following (FOLLOW): it takes
// mt's fraction, so that the tile's largest key, a whole number of units away,
// has P = a power of two, which bf16 holds without rounding. It keeps its whole
// part, one above that of the score it was last raised to, so it is always
// above that score: in either mode P stays below 2^8 and the accumulators
// below 2^8 times the sum of what they hold, however the tiles' maxima fall.
template <bool FOLLOW>
__device__ __forceinline__ float next_ref(float mt, float m_run, bool grow) {
  if constexpr (!FOLLOW) return grow ? mt : m_run;
  const float whole = floorf(m_run);
  const float t = whole + __builtin_amdgcn_fractf(mt);
  const float moved = t - whole < 1.f ? t : whole;  // (a sum that was rounded up)
  return grow ? mt + 1.f : mt == kNegInf ? m_run : moved;
}

// Waves per SIMD the register allocation must allow: three for one row block
// (168 registers), else two (256). Two groups of three blocks at D = 128 use all
// 256 and keep three or four values in scratch that the ring's loop reads back
// (six loads per round of four tiles).
template <int D, int NQ, int QG, bool NT, bool FOLLOW, bool WIN>
__global__ void __launch_bounds__(Shape<QG>::kThreads, NQ == 1 && QG == 1 ? 3 : 2)
attn_split_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ kc,
                  const uint16_t* __restrict__ vc, const uint8_t* __restrict__ mask,
                  const int32_t* __restrict__ kv_len, const int32_t* __restrict__ gamma,
                  void* __restrict__ out, bool out_bf16, float* __restrict__ part_o,
                  float* __restrict__ part_ml, uint32_t* __restrict__ counters,
                  const int32_t* __restrict__ order, int B, int gmax, int Hq, int Hkv, int L_cap,
                  int window, int sinks, float scale_log2, int split_keys, int n_splits, int q_chunks,
                  int32_t* __restrict__ status) {
  using GG = Geo<D>;
  constexpr int MQ = 16 * NQ;
  constexpr int DB = D / 16;
  constexpr int kT = Shape<QG>::kThreads;
  constexpr int kRing = Shape<QG>::kRing;
  constexpr int kBufs = Shape<QG>::kBufs;
  constexpr int kLd = GG::kLoads / QG;  // 16-byte loads per lane per tensor per tile
  __shared__ __attribute__((aligned(16))) unsigned char lds[Lds<D, NQ, QG>::kBytes];

  // Workgroup order: with an order table (more workgroups than fit on the
  // device at once), the table's: jobs by decreasing key count, so that the
  // last workgroups to start are the shortest. Otherwise (sequence, kv head)
  // pair fastest, then key split in descending order, then query chunk.
  // Workgroups are dealt to the XCDs round-robin, so each XCD gets every
  // split of an even share of the pairs (and the query chunks of one pair and
  // split share an XCD and its L2).
  const int P = B * Hkv;
  const int rest = (int)(blockIdx.x / (unsigned)P);
  const int code = order ? __builtin_amdgcn_readfirstlane(order[blockIdx.x])
                         : ((int)(blockIdx.x % (unsigned)P) * q_chunks + rest / n_splits) * n_splits +
                               (n_splits - 1 - rest % n_splits);
  const int split = code % n_splits;
  const int job = code / n_splits;
  const int qc = job % q_chunks;
  const int pair_id = job / q_chunks;
  const int g = pair_id % Hkv;
  const int b = pair_id / Hkv;
  const int G = Hq / Hkv;
  const int R = G * (gmax + 1);
  const int gam = gamma[b];
  const int L = kv_len[b];
  const bool valid = gam >= 0 && gam <= gmax && L >= gam + 1 && L <= L_cap;
  if (!valid && split == 0 && qc == 0 && g == 0 && threadIdx.x == 0 && status) {
    atomicOr(status, (gam < 0 || gam > gmax) ? SR_ST_GAMMA : SR_ST_KVLEN);
  }
  const int row0 = qc * QG * MQ;
  const int row_end = min(R, row0 + QG * MQ);
  const int Mb = valid ? G * (gam + 1) : 0;
  const Reach<kWaveKeys> reach(WIN && valid ? L - gam - 1 : 0, WIN && valid ? L : 0, WIN ? window : 1, WIN ? sinks : 0);
  const int n_keys = !valid ? 0 : WIN ? reach.tiles * kWaveKeys : L;
  const int ns = (n_keys + split_keys - 1) / split_keys;  // splits that hold keys
  const bool work = row0 < Mb && split < ns;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = wave_id();
  const int ws = w % kWaves;  // key stream
  const int h = w / kWaves;   // query group: rows rbase .. rbase + MQ - 1
  const int rbase = row0 + h * MQ;
  const int l16 = lane & 15;
  const int lg = lane >> 4;

  // Four columns of output row r. Without a window the output is fp32; with one,
  // fp32 or bf16 (rounded once, from the 32-bit sums).
  auto store = [&](int r, int col, const floatx4& x) __attribute__((always_inline)) {
    const int i = r / G, hh = g * G + r % G;
    const size_t at = ((size_t)(b * (gmax + 1) + i) * Hq + hh) * D + col;
    if (WIN && out_bf16) *(u32x2*)((uint16_t*)out + at) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    else *(floatx4*)((float*)out + at) = x;
  };
  if (!work) {
    // Nothing to compute. Split 0 of a query chunk without live rows (or of an
    // invalid sequence) owns those output rows and writes them as zero.
    if (split == 0) {
      for (int idx = tid; idx < (row_end - row0) * (D / 4); idx += kT) {
        const int r = row0 + idx / (D / 4);
        const int d4 = idx % (D / 4);
        store(r, d4 * 4, floatx4{0.f, 0.f, 0.f, 0.f});
      }
    }
    return;
  }

  unsigned char* qst = lds + kWaves * kBufs * GG::kWaveBytes;
  const size_t slab = ((size_t)b * Hkv + g) * (size_t)L_cap;
  const uint16_t* kslab = kc + slab * D;
  const uint16_t* vslab = vc + slab * D;
  const uint8_t* mrow = mask ? mask + (size_t)b * L_cap : nullptr;
  const int causal0 = L - gam - 1;  // cache position of new row 0

  floatx4 o[DB][NQ];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int qg = 0; qg < NQ; ++qg) {
    m_run[qg] = kNegInf;
    l_run[qg] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qg] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // Tile j holds keys [16 j, 16 j + 16). Split s owns the keys
  // [s split_keys, (s + 1) split_keys), dealt round-robin to the four
  // streams, so a stream's tiles are first, first + 4, first + 8, ... below
  // j_end.
  const int first0 = split * (split_keys / kWaveKeys);
  const int first = first0 + ws;
  const int j_end = min(WIN ? reach.tiles : (L + kWaveKeys - 1) / kWaveKeys, (split + 1) * (split_keys / kWaveKeys));
  const int row_lim = WIN ? L : min(L, j_end * kWaveKeys);  // a refill past the stream's last tile reads nothing
  // First key of tile j (with a window, past the stream's last tile: a row that is never read).
  auto tile_key = [&](int j) __attribute__((always_inline)) {
    return !WIN ? j * kWaveKeys : j < j_end ? reach.start(j) : L;
  };
  // Whether some row sees key k, and whether every row sees the tile from key k on (but for the causal limit)
  auto in_reach = [&](int k) __attribute__((always_inline)) { return !WIN || k >= reach.first_key || k < sinks; };
  auto all_see = [&](int k) __attribute__((always_inline)) { return !WIN || k > L - 1 - window || k + kWaveKeys <= sinks; };
  // Whether the row whose last key is lim sees key k <= lim
  auto in_window = [&](int k, int lim) __attribute__((always_inline)) { return !WIN || k > lim - window || k < sinks; };

  // Every fetch issues the same loads (rows at or past kv_len, and tiles past
  // the stream's last, read out of range, as zero, with no traffic), so each
  // wait covers exactly the loads it needs, in the first iteration as in
  // every later one.
  const uint8_t* mload = mrow ? mrow : (const uint8_t*)kslab;
  // K/V slabs of (b, g) as buffer resources: 32-bit row offsets
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(kslab, (size_t)L_cap * D * 2);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(vslab, (size_t)L_cap * D * 2);
  const int lane_row = lane / GG::kChunksPerRow;
  const int lane_chunk = lane % GG::kChunksPerRow;
  const uint32_t lane_col = (uint32_t)lane_chunk * 16;
  // this wave's rows of a tile: load u covers rows (h kLd + u) kRowsPerLoad + lane_row
  auto fetch = [&](int j, Stage<D, QG>& st) __attribute__((always_inline)) {
    const int kb0 = tile_key(j);
#pragma unroll
    for (int u = 0; u < kLd; ++u) {
      const int row = kb0 + (h * kLd + u) * GG::kRowsPerLoad + lane_row;
      const uint32_t off = row < row_lim ? (uint32_t)row * (D * 2) + lane_col : kOutOfRange;
      st.k[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, off, 0, NT ? kStreamLoad : 0));
      st.v[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, NT ? kStreamLoad : 0));
    }
    st.mbyte = mload[min(kb0 + (lane & (kWaveKeys - 1)), L - 1)];
  };
  // With a window: P of the scores score(qg, e), e < N, of a row's N keys per lane,
  // two at a time to put(qg, pair, bf16x2). Lazy, a row's reference stands until a score
  // exceeds it by more than 2^kLazy; only then do its four lanes need their common
  // maximum. Each lane sums its own keys; the row's lanes are added up at the end.
  auto window_softmax = [&](auto blocks, auto score, auto count, auto put) __attribute__((always_inline)) {
    constexpr int NL = decltype(blocks)::value;
    constexpr int N = decltype(count)::value;
    float mt[NL];
    bool over = false;
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) {
      mt[qg] = kNegInf;
#pragma unroll
      for (int e = 0; e < N; ++e) mt[qg] = fmaxf(mt[qg], score(qg, e));
      mt[qg] *= scale_log2;
      over |= mt[qg] > m_run[qg] + kLazy;
    }
    if (FOLLOW || rare(__ballot(over) != 0ull)) {
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) {
        const float m = max_across_rows(mt[qg]);
        const float mref = next_ref<FOLLOW>(m, m_run[qg], m > m_run[qg] + (FOLLOW ? kLazyFollow : kLazy));
        const float alpha = m_run[qg] == mref ? 1.f : exp2_hw(m_run[qg] - mref);
        m_run[qg] = mref;
        l_run[qg] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db][qg] *= alpha;
      }
    }
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) {
      const float mr = m_run[qg] == kNegInf ? 0.f : m_run[qg];  // (-inf: no key of the row so far)
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float p0 = exp2_hw(fmaf(score(qg, e), scale_log2, -mr));
        const float p1 = exp2_hw(fmaf(score(qg, e + 1), scale_log2, -mr));
        l_run[qg] += p0;
        l_run[qg] += p1;
        put(qg, e / 2, to_bf16x2(p0, p1));
      }
    }
  };
  // One query group. Ring entry st holds tile j: stage it in the stream's slot,
  // refill it with the stream's tile kRing further on, compute tile j, and
  // leave the refilled tile's number in j.
  // With a window, for the first NL of the wave's row blocks (the others hold no live row).
  auto step = [&](auto blocks, int& j, Stage<D, QG>& st) __attribute__((always_inline)) {
    constexpr int NL = decltype(blocks)::value;
    unsigned char* kst = lds + ws * kBufs * GG::kWaveBytes;
    unsigned char* vst = kst + GG::kSlotK;
    const int kb0 = tile_key(j);
    const bool key_ok = lane < kWaveKeys && kb0 + lane < L && in_reach(kb0 + lane) && (mrow == nullptr || st.mbyte != 0u);
    const uint32_t vbits = (uint32_t)__ballot(key_ok) & 0xffffu;
    const bool all_rows = vbits == 0xffffu;  // wave-uniform
#pragma unroll
    for (int u = 0; u < kLd; ++u) {
      const int rl = (h * kLd + u) * GG::kRowsPerLoad + lane_row;
      *(u32x4*)(kst + rl * GG::kKStride + lane_chunk * 16) = st.k[u];
      const u32x4 vv = (all_rows || ((vbits >> rl) & 1u)) ? st.v[u] : u32x4{0u, 0u, 0u, 0u};
      uint32_t* dst = (uint32_t*)(vst + rl * GG::kVStride + lane_chunk * 16);
      *(uint2*)dst = make_uint2(vv.x, vv.y);
      *(uint2*)(dst + 2) = make_uint2(vv.z, vv.w);
    }
    wave_lds_sync();
    const int nx = j + kRing * kWaves;
    __builtin_amdgcn_sched_barrier(0);
    fetch(nx, st);  // the ring's other tiles and this refill stay in flight during the compute below
    __builtin_amdgcn_sched_barrier(0);
    const int jc = j;
    j = nx;
    if (jc >= j_end || rbase >= Mb) return;  // wave-uniform: past the stream's last tile, or no live rows
    const bool full = vbits == 0xffffu && kb0 + kWaveKeys - 1 <= causal0 && all_see(kb0);  // wave-uniform
    // ---- S^T = K Q^T (16 keys x 16 queries per block)
    floatx4 sacc[NL];
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) sacc[qg] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const int col = (ks * 32 + lg * 8) * 2;
      const bf16x8 ka = *(const bf16x8*)(kst + l16 * GG::kKStride + col);
      bf16x8 qb[NL];
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) qb[qg] = *(const bf16x8*)(qst + (h * MQ + qg * 16 + l16) * GG::kKStride + col);
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) sacc[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[qg], sacc[qg], 0, 0, 0);
    }
    // ---- mask, online softmax, P in bf16 (lane: keys lg*4 + e of query l16)
    // Row blocks without live rows go through both products too (on zero
    // query rows and zero P): a branch around each MFMA costs more than the
    // MFMA. Only the softmax is skipped for them.
    shortx4 pb[NL];
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) pb[qg] = shortx4{0, 0, 0, 0};
    if constexpr (WIN) {
      if (rare(!full)) {
        int r16 = l16, r4 = lg * 4;  // (hidden from the optimiser, which would keep what follows from them in registers)
        asm volatile("" : "+v"(r16), "+v"(r4));
#pragma unroll
        for (int qg = 0; qg < NL; ++qg) {
          const int r = rbase + qg * 16 + r16;
          const int lim = r < Mb ? causal0 + r / G : -1;  // last key this query row sees
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = kb0 + r4 + e;
            const bool vis = (((vbits >> (r4 + e)) & 1u) != 0u) & (k <= lim) & in_window(k, lim);
            sacc[qg][e] = vis ? sacc[qg][e] : kNegInf;
          }
        }
      }
      window_softmax(blocks, [&](int qg, int e) __attribute__((always_inline)) { return sacc[qg][e]; },
                     std::integral_constant<int, 4>{},
                   [&](int qg, int pair, uint32_t two) __attribute__((always_inline)) {
                     u32x2 w = __builtin_bit_cast(u32x2, pb[qg]);
                     w[pair] = two;
                     pb[qg] = __builtin_bit_cast(shortx4, w);
                   });
    } else {
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) {
      if (rbase + qg * 16 < Mb) {
        const int r = rbase + qg * 16 + l16;
        float s[4];
        float mt = kNegInf;
        if (full) {
          // every row of the wave sees all 16 keys (rows past Mb are dropped
          // at the end); the scale is positive, so the maximum is taken on the
          // raw products and each probability below is one fma and one exp2
          mt = fmaxf(fmaxf(sacc[qg][0], sacc[qg][1]), fmaxf(sacc[qg][2], sacc[qg][3])) * scale_log2;
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = sacc[qg][e];
        } else {
          const int lim = r < Mb ? causal0 + r / G : -1;  // last key this query row sees
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int kl = lg * 4 + e;
            const bool vis = ((vbits >> kl) & 1u) && (kb0 + kl <= lim);
            s[e] = vis ? sacc[qg][e] * scale_log2 : kNegInf;
            mt = fmaxf(mt, s[e]);
          }
        }
        mt = max_across_rows(mt);
        // P stays below 2^kLazy; the output accumulators are rescaled only
        // when the reference moves (skipped by the whole wave when no row's does).
        // (straight-line: every exponential is computed and selected, no
        // per-entry branches)
        const bool grow = mt > m_run[qg] + (FOLLOW ? kLazyFollow : kLazy);
        const float mref = next_ref<FOLLOW>(mt, m_run[qg], grow);
        // exp2(-inf) = 0 covers a first reference (the old one -inf); equal
        // references, -inf ones included, give 1
        const float alpha = m_run[qg] == mref ? 1.f : exp2_hw(m_run[qg] - mref);
        const float mr = mref == kNegInf ? 0.f : mref;  // (-inf: every score of the row so far is -inf)
        float pk[4];
        float ls = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pk[e] = exp2_hw(full ? fmaf(s[e], scale_log2, -mr) : s[e] - mr);
          ls += pk[e];
        }
        ls = sum_across_rows(ls);
        l_run[qg] = l_run[qg] * alpha + ls;
        m_run[qg] = mref;
        if (FOLLOW || __ballot(grow) != 0ull) {
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db][qg] *= alpha;
        }
        const uint32_t w0 = pack_bf16x2(pk[0], pk[1]);
        const uint32_t w1 = pack_bf16x2(pk[2], pk[3]);
        pb[qg] = __builtin_bit_cast(shortx4, make_uint2(w0, w1));
      }
    }
    }
    // ---- O^T += V^T P^T (K = 16 keys)
    // The V^T operand (lane: column l16 of the block, keys lg*4 .. lg*4+3) by
    // the LDS transposing read: in each 16-lane group, lane j names the four
    // columns 4 (j mod 4) .. +3 of key row lg*4 + j/4, and lane i receives
    // column i of the group's four key rows.
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const unsigned char* vrow = vst + (lg * 4 + (l16 >> 2)) * GG::kVStride + (db * 16 + (l16 & 3) * 4) * 2;
      const shortx4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)vrow);
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) {
        o[db][qg] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(va, pb[qg], o[db][qg], 0, 0, 0);
      }
    }
    wave_lds_sync();  // this tile's LDS reads are issued before the slot is rewritten
  };

  // Two query groups: two of the stream's tiles at a time. Both are staged (one
  // LDS buffer each), the query fragments of a k-step are read once for both, the
  // softmax of a row takes its 32 keys together (one maximum and one sum across
  // lanes), and the second product runs over 32 keys per instruction: its k
  // slots lg*8 + e hold the first tile's key lg*4 + e (e < 4) and the second's
  // lg*4 + e - 4, which is how the scores and the transposed V reads lie in the
  // registers. (One tile at a time, 16 keys per instruction: 127 us at 4
  // sequences of 32768 keys, 72 query rows per KV head; now 119.)
  auto step2 = [&](auto blocks, int& ja, Stage<D, QG>& sa, int& jb, Stage<D, QG>& sb) __attribute__((always_inline)) {
    constexpr int NL = decltype(blocks)::value;
    unsigned char* kst = lds + (ws * kBufs) * GG::kWaveBytes;
    uint32_t vb[2];
    auto stage = [&](int j, Stage<D, QG>& st, int buf) __attribute__((always_inline)) {
      unsigned char* kd = kst + buf * GG::kWaveBytes;
      unsigned char* vd = kd + GG::kSlotK;
      const int kb0 = tile_key(j);
      const bool key_ok =
          lane < kWaveKeys && j < j_end && kb0 + lane < L && in_reach(kb0 + lane) && (mrow == nullptr || st.mbyte != 0u);
      const uint32_t vbits = (uint32_t)__ballot(key_ok) & 0xffffu;
      const bool all_rows = vbits == 0xffffu;  // wave-uniform
#pragma unroll
      for (int u = 0; u < kLd; ++u) {
        const int rl = (h * kLd + u) * GG::kRowsPerLoad + lane_row;
        *(u32x4*)(kd + rl * GG::kKStride + lane_chunk * 16) = st.k[u];
        const u32x4 vv = (all_rows || ((vbits >> rl) & 1u)) ? st.v[u] : u32x4{0u, 0u, 0u, 0u};
        uint32_t* dst = (uint32_t*)(vd + rl * GG::kVStride + lane_chunk * 16);
        *(uint2*)dst = make_uint2(vv.x, vv.y);
        *(uint2*)(dst + 2) = make_uint2(vv.z, vv.w);
      }
      return vbits;
    };
    vb[0] = stage(ja, sa, 0);
    vb[1] = stage(jb, sb, 1);
    __syncthreads();  // both halves of both tiles are in the slot
    const int j0 = ja, j1 = jb;
    ja += kRing * kWaves;
    jb += kRing * kWaves;
    __builtin_amdgcn_sched_barrier(0);
    fetch(ja, sa);  // these and the ring's other tiles stay in flight during the compute below
    fetch(jb, sb);
    __builtin_amdgcn_sched_barrier(0);
    if (j0 < j_end && rbase < Mb) {  // wave-uniform
      const int kb[2] = {tile_key(j0), tile_key(j1)};
      const bool full = (vb[0] & vb[1]) == 0xffffu && kb[1] + kWaveKeys - 1 <= causal0 && all_see(kb[0]) && all_see(kb[1]);  // wave-uniform
      floatx4 sacc[2][NL];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int qg = 0; qg < NL; ++qg) sacc[t][qg] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const int col = (ks * 32 + lg * 8) * 2;
        bf16x8 qb[NL];
#pragma unroll
        for (int qg = 0; qg < NL; ++qg) qb[qg] = *(const bf16x8*)(qst + (h * MQ + qg * 16 + l16) * GG::kKStride + col);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bf16x8 ka = *(const bf16x8*)(kst + t * GG::kWaveBytes + l16 * GG::kKStride + col);
#pragma unroll
          for (int qg = 0; qg < NL; ++qg) sacc[t][qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[qg], sacc[t][qg], 0, 0, 0);
        }
      }
      bf16x8 pb[NL];
      if constexpr (WIN) {
        if (rare(!full)) {
          int r16 = l16, r4 = lg * 4;
          asm volatile("" : "+v"(r16), "+v"(r4));
#pragma unroll
          for (int qg = 0; qg < NL; ++qg) {
            const int r = rbase + qg * 16 + r16;
            const int lim = r < Mb ? causal0 + r / G : -1;  // last key this query row sees
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int kl = r4 + e % 4;
              const int k = kb[e / 4] + kl;
              const bool vis = (((vb[e / 4] >> kl) & 1u) != 0u) & (k <= lim) & in_window(k, lim);
              sacc[e / 4][qg][e % 4] = vis ? sacc[e / 4][qg][e % 4] : kNegInf;
            }
          }
        }
        window_softmax(blocks, [&](int qg, int e) __attribute__((always_inline)) { return sacc[e / 4][qg][e % 4]; },
                     std::integral_constant<int, 8>{},
                     [&](int qg, int pair, uint32_t two) __attribute__((always_inline)) {
                       u32x4 w = __builtin_bit_cast(u32x4, pb[qg]);
                       w[pair] = two;
                       pb[qg] = __builtin_bit_cast(bf16x8, w);
                     });
      } else {
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) {
        pb[qg] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
        if (rbase + qg * 16 < Mb) {
          const int r = rbase + qg * 16 + l16;
          float sc[8];
          float mt = kNegInf;
          if (full) {  // every row sees all 32 keys (see the single-tile step)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              sc[e] = sacc[e / 4][qg][e % 4];
              mt = fmaxf(mt, sc[e]);
            }
            mt *= scale_log2;
          } else {
            const int lim = r < Mb ? causal0 + r / G : -1;  // last key this query row sees
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int kl = lg * 4 + e % 4;
              const int kb0 = (e < 4 ? j0 : j1) * kWaveKeys;
              const bool vis = ((vb[e / 4] >> kl) & 1u) && (kb0 + kl <= lim);
              sc[e] = vis ? sacc[e / 4][qg][e % 4] * scale_log2 : kNegInf;
              mt = fmaxf(mt, sc[e]);
            }
          }
          mt = max_across_rows(mt);
          const bool grow = mt > m_run[qg] + (FOLLOW ? kLazyFollow : kLazy);
          const float mref = next_ref<FOLLOW>(mt, m_run[qg], grow);
          const float alpha = m_run[qg] == mref ? 1.f : exp2_hw(m_run[qg] - mref);
          const float mr = mref == kNegInf ? 0.f : mref;
          float pk[8];
          float ls = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            pk[e] = exp2_hw(full ? fmaf(sc[e], scale_log2, -mr) : sc[e] - mr);
            ls += pk[e];
          }
          ls = sum_across_rows(ls);
          l_run[qg] = l_run[qg] * alpha + ls;
          m_run[qg] = mref;
          if (FOLLOW || __ballot(grow) != 0ull) {
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db][qg] *= alpha;
          }
          pb[qg] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(pk[0], pk[1]), pack_bf16x2(pk[2], pk[3]),
                                                    pack_bf16x2(pk[4], pk[5]), pack_bf16x2(pk[6], pk[7])});
        }
      }
      }
      typedef short shortx8 __attribute__((ext_vector_type(8)));
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const unsigned char* vrow = kst + GG::kSlotK + (lg * 4 + (l16 >> 2)) * GG::kVStride + (db * 16 + (l16 & 3) * 4) * 2;
        const shortx4 va0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)vrow);
        const shortx4 va1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(vrow + GG::kWaveBytes));
        const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(va0, va1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int qg = 0; qg < NL; ++qg) o[db][qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[qg], o[db][qg], 0, 0, 0);
      }
    }
    __syncthreads();  // every read of the two buffers came before the next tiles
  };

  // Issue order: this workgroup's query rows, then the ring; the query rows
  // are staged in LDS while the K/V tiles are still in flight. Each group is
  // kept together (no interleaving by the scheduler), so every wait covers
  // exactly what it needs: a step waits for its own tile only.
  constexpr int kQChunks = QG * MQ * GG::kChunksPerRow;
  constexpr int kQLoads = (kQChunks + kT - 1) / kT;
  u32x4 qv[kQLoads];
#pragma unroll
  for (int u = 0; u < kQLoads; ++u) {
    const int idx = min(tid + u * kT, kQChunks - 1);
    const int r = min(row0 + idx / GG::kChunksPerRow, Mb - 1);  // rows past Mb are zeroed below
    const int i = r / G, hh = g * G + r % G;
    qv[u] = *(const u32x4*)(q + ((size_t)(b * (gmax + 1) + i) * Hq + hh) * D + (idx % GG::kChunksPerRow) * 8);
  }
  __builtin_amdgcn_sched_barrier(0);
  Stage<D, QG> ring[kRing];
  int jr[kRing];
#pragma unroll
  for (int r = 0; r < kRing; ++r) {
    jr[r] = first + r * kWaves;
    fetch(jr[r], ring[r]);
    __builtin_amdgcn_sched_barrier(0);
  }
  // (unconditional: a thread past the last chunk rewrites that chunk with
  // the same value, and no load is moved into a branch after the K/V loads)
#pragma unroll
  for (int u = 0; u < kQLoads; ++u) {
    const int idx = min(tid + u * kT, kQChunks - 1);
    const int rl = idx / GG::kChunksPerRow;
    const u32x4 val = row0 + rl < Mb ? qv[u] : u32x4{0u, 0u, 0u, 0u};
    *(u32x4*)(qst + rl * GG::kKStride + (idx % GG::kChunksPerRow) * 16) = val;
  }
  __syncthreads();

  // The ring holds the stream's next kRing tiles (ascending). With two query
  // groups every wave runs the same number of rounds (counted on stream 0,
  // whose tiles come first), so the barriers inside the steps pair up; a step
  // past a stream's last tile still stages (zeros) and meets the barrier.
  if constexpr (WIN) {
    auto loop = [&](auto blocks) __attribute__((always_inline)) {
      if constexpr (QG == 1) {
        while (jr[0] < j_end) {
  #pragma unroll
          for (int r = 0; r < kRing; ++r) step(blocks, jr[r], ring[r]);
        }
      } else {
        const int rounds = (j_end - first0 + kRing * kWaves - 1) / (kRing * kWaves);
        for (int it = 0; it < rounds; ++it) {
  #pragma unroll
          for (int r = 0; r < kRing; r += 2) step2(blocks, jr[r], ring[r], jr[r + 1], ring[r + 1]);
        }
      }
    };
    // (with two groups the copies of the loop for fewer blocks would take registers
    // from each other: 4096-position windows of 16 sequences, 72 rows, 81 us with them,
    // 67 without)
    const int live = QG == 2 ? NQ : min(NQ, (Mb - rbase + 15) / 16);
    if (NQ >= 3 && live >= 3) loop(std::integral_constant<int, NQ >= 3 ? 3 : 1>{});
    else if ((QG == 1 || NQ == 2) && NQ >= 2 && live >= 2) loop(std::integral_constant<int, NQ >= 2 ? 2 : 1>{});
    else if (QG == 1) loop(std::integral_constant<int, 1>{});
#pragma unroll
    for (int qg = 0; qg < NQ; ++qg) l_run[qg] = sum_across_rows(l_run[qg]);
  } else if constexpr (QG == 1) {
    while (jr[0] < j_end) {
#pragma unroll
      for (int r = 0; r < kRing; ++r) step(std::integral_constant<int, NQ>{}, jr[r], ring[r]);
    }
  } else {
    const int rounds = (j_end - first0 + kRing * kWaves - 1) / (kRing * kWaves);
    for (int it = 0; it < rounds; ++it) {
#pragma unroll
      for (int r = 0; r < kRing; r += 2)
        step2(std::integral_constant<int, NQ>{}, jr[r], ring[r], jr[r + 1], ring[r + 1]);
    }
  }
  __syncthreads();

  const JobRows J{row0, row_end, Mb, R, split, ns, n_splits, job, P, (size_t)(b * Hkv + g)};
  merge_and_store<MergeLds<D, NQ, QG>, D, NQ, QG, Lds<D, NQ, QG>::kBytes, WIN>(
      lds, o, m_run, l_run, J, part_o, part_ml, counters, store);
}

template <int D, bool FOLLOW, bool WIN>
SplitKernel pick_split(int nq, int qg, int q_chunks) {
  if (qg == 1) {
    switch (nq) {
      case 1: return attn_split_kernel<D, 1, 1, true, FOLLOW, WIN>;
      case 2: return !WIN || q_chunks == 1 ? attn_split_kernel<D, 2, 1, true, FOLLOW, WIN>
                                           : attn_split_kernel<D, 2, 1, !WIN, FOLLOW, WIN>;
      default: return !WIN || q_chunks == 1 ? attn_split_kernel<D, 3, 1, true, FOLLOW, WIN>
                                            : attn_split_kernel<D, 3, 1, !WIN, FOLLOW, WIN>;
    }
  }
  if (nq == 2) return attn_split_kernel<D, 2, 2, true, FOLLOW, WIN>;
  return q_chunks == 1 ? attn_split_kernel<D, 3, 2, true, FOLLOW, WIN> : attn_split_kernel<D, 3, 2, false, FOLLOW, WIN>;
}

}  // namespace
}  // namespace sr
