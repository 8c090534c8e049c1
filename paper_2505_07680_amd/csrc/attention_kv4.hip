// Verification attention over a K/V cache held in 4 bits (gfx950): the
// attention of the new rows (Section 2.2 step 2; Section 4.4, Eq. 8), with or
// without a window, over e2m1 codes with a power of two per 32 elements of a row.
//
// Work decomposition as over a bf16 cache: a workgroup of four waves takes one
// (sequence, kv head, query chunk, key split; small batches split by their lengths,
// see deal), the waves deal the split's tiles of 32 keys among themselves, and their states merge through LDS, those of
// several splits through the workspace.
//
// A code times its power is exact in bf16, so both products run on bf16 MFMA and
// the only roundings are those of the bf16 attention (P, and the output's).
// The hardware widens two codes per instruction and scales them on the way
// (v_cvt_scalef32_pk_bf16_fp4). Per 32-key tile of a wave, lane (l16, lg):
//   * K: lane l16 of quarter lg takes a quarter of the key's row (D/4 codes, one
//     16-byte load at D = 128), which all lie under one power. Widened, they are
//     the A operand of S^T = K Q^T as they stand: the contraction over the head
//     dimension takes its elements in the order (ks, lg, e) -> lg D/4 + 8 ks + e,
//     and the query rows, which stay in registers, are held in the same order. K
//     never passes through LDS.
//   * V: the same load, widened and written to the wave's own LDS slot row by row
//     (rows that no query sees as zeros), to come back transposed
//     (ds_read_b64_tr_b16) as the A operand of O^T += V^T P^T over 32 keys. The
//     16-byte chunks of a row are permuted by the row's number, so that neither
//     the writes (eight rows at a time) nor the transposing reads (four) meet in
//     a bank.
//   * softmax as over bf16 with lazy references: a row's is raised only when a tile
//     exceeds it by more than 2^8, P rounds to bf16. (1.4e-3 to 1.6e-3 of the values off
//     the 64-bit result. References that follow the tiles, which the bf16 attention has
//     for small batches, come to 1.0e-3 and would rescale the accumulators every tile.)
//
// With one query row per head HBM bounds it (256 sequences of 4096 keys, 32/8
// heads of 128: 179 to 198 us, 5.8 to 6.4 TB/s); with more rows the instructions of
// two waves per SIMD do: 256 of 256 to 8192 keys, gamma 1 to 8, 242 us, 5.0 TB/s,
// vector units 47% busy, matrix units 24%, LDS 30% (over a bf16 cache 730 us). 16
// sequences of 2048, gamma 5, take 19 us, half of it latency: start, lengths and
// first loads before the loop, the merge of four splits after it.

#include <type_traits>

#include "attention_common.h"

namespace sr {
namespace {

constexpr int kTile = 32;   // keys per tile of a wave
constexpr int kMaxNQ4 = 3;  // 16-row query blocks per wave: more than 48 rows go to further query chunks
constexpr int kMergeMost4 = 49152;  // the merge's LDS: three workgroups fit a CU's
constexpr int kRegNQ = 2;   // of them with their query rows in registers

template <int D, int NQ>
struct Lds4 {
  static constexpr int kRow = D * 2;               // bytes of a widened V row
  static constexpr int kSlot = kTile * kRow;       // a tile's V, per wave
  static constexpr int kReg = NQ < 3 ? NQ : kRegNQ;
  static constexpr int kQRows = 16 * (NQ - kReg);  // query rows that stay here
  static constexpr int kQ = kWaves * kSlot;
  static constexpr int kStage = kQ + kQRows * D * 2;
  using Merge = MergeLds<D, NQ, 1, kMergeMost4>;
  static constexpr int kComb = Merge::kComb;
  static constexpr int kBytes = kStage > kComb ? kStage : kComb;
};

// Eight codes (one dword) times 2^(p - 127), `scale` that power as a float.
__device__ __forceinline__ u32x4 widen(uint32_t codes, float scale) {
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return v;
}

// Where 16-byte chunk c of V row r sits in its row.
__device__ __forceinline__ int chunk_at(int c, int r) { return c ^ (((r & 3) << 1) | ((r >> 2) & 1)); }

template <int D>
struct Stage4 {  // a 32-key tile in flight: rows u 16 + l16
  uint32_t k[2][D / 32], v[2][D / 32];
  uint8_t kp[2], vp[2];
  uint8_t mbyte;
  int key;         // first key
};

struct Kv4Args {
  const uint16_t* q;
  const uint8_t *kc, *kp, *vc, *vp;
  const uint8_t* mask;
  const int32_t *kv_len, *gamma;
  void* out;
  bool out_bf16;
  float *part_o, *part_ml;
  uint32_t* counters;
  const int32_t* order;
  int B, gmax, Hq, Hkv, L_cap, window, sinks;
  float scale_log2;
  int split_keys, n_splits, q_chunks, units;
  int32_t* status;
};

// Of 32-bit lane values: their sum and maximum over the wave, and the sums up to each lane.
__device__ __forceinline__ int over_rows(int x, int row) { return __builtin_amdgcn_readlane(x, row * 16); }
__device__ __forceinline__ int wave_sum_i(int x) {
  x += (int)perm_u32<dpp::kXor1>((uint32_t)x);
  x += (int)perm_u32<dpp::kXor2>((uint32_t)x);
  x += (int)perm_u32<dpp::kHalfMirror>((uint32_t)x);
  x += (int)perm_u32<dpp::kMirror>((uint32_t)x);
  return over_rows(x, 0) + over_rows(x, 1) + over_rows(x, 2) + over_rows(x, 3);
}
__device__ __forceinline__ int wave_max_i(int x) {
  x = max(x, (int)perm_u32<dpp::kXor1>((uint32_t)x));
  x = max(x, (int)perm_u32<dpp::kXor2>((uint32_t)x));
  x = max(x, (int)perm_u32<dpp::kHalfMirror>((uint32_t)x));
  x = max(x, (int)perm_u32<dpp::kMirror>((uint32_t)x));
  return max(max(over_rows(x, 0), over_rows(x, 1)), max(over_rows(x, 2), over_rows(x, 3)));
}
template <int N>
__device__ __forceinline__ int row_shr(int x) {  // lane i: lane i - N of its row of 16, or 0
  return __builtin_amdgcn_update_dpp(0, x, 0x110 + N, 0xf, 0xf, true);
}
__device__ __forceinline__ int wave_scan_i(int x) {
  x += row_shr<1>(x);
  x += row_shr<2>(x);
  x += row_shr<4>(x);
  x += row_shr<8>(x);
  const int r0 = __builtin_amdgcn_readlane(x, 15), r1 = __builtin_amdgcn_readlane(x, 31);
  const int r2 = __builtin_amdgcn_readlane(x, 47), row = (int)(threadIdx.x & 63) / 16;
  return x + (row > 0 ? r0 : 0) + (row > 1 ? r1 : 0) + (row > 2 ? r2 : 0);
}

// The work of a launch dealt by the lengths (up to 64 sequences, one per lane):
// splits of one size for all, the least (to within 1/32, where the search for it stops)
// that gives no more (sequence, split) pairs than there is room for, but not below
// what a merge costs (a split of K keys and its share of the merge take K + 64 L / K,
// least at K = sqrt(64 L)). Unit s of the launch is split s - first of sequence b;
// every wave finds the same.
constexpr int kMaxDealt = 64;
constexpr int kMergeKeys = 64;  // keys that a merged split's time is worth
struct Dealt {
  int b, first, tiles;  // sequence, its first unit, tiles per split
  bool any;
  int gam, L;
};
inline __host__ __device__ int least_tiles(int tiles) {
  return tiles * kTile <= 4 * kMergeKeys ? tiles : (int)ceilf(sqrtf((float)tiles * ((float)kMergeKeys / kTile)));
}
__device__ __forceinline__ Dealt deal(const Kv4Args& a, int window, int s) {
  const int lane = threadIdx.x & 63;
  const int lb = min(lane, a.B - 1);
  const int gam = a.gamma[lb], L = a.kv_len[lb];
  const bool valid = gam >= 0 && gam <= a.gmax && L >= gam + 1 && L <= a.L_cap;
  const Reach<kTile> reach(valid ? L - gam - 1 : 0, valid ? L : 0, window, a.sinks);
  const int tiles = lane < a.B ? max(reach.tiles, 1) : 0;  // (bad data: one split, which writes zeros)
  const int most = wave_max_i(tiles), total = wave_sum_i(tiles);
  auto splits = [&](int size) __attribute__((always_inline)) { return (int)((uint32_t)(tiles + size - 1) / (uint32_t)size); };
  int lo = min(max(least_tiles(most), (total + a.units - 1) / a.units), most), hi = most;  // (hi: one split each)
  if (wave_sum_i(splits(lo)) <= a.units) {
    hi = lo;
  } else {
    const int room = a.units - a.B;  // sum ceil(t / size) < total / size + B
    if (room > 0) hi = min(hi, (total + room - 1) / room);
    while (hi - lo > 1 + lo / 32) {
      const int mid = (lo + hi) / 2;
      if (wave_sum_i(splits(mid)) <= a.units) hi = mid;
      else lo = mid;
    }
  }
  const int n = splits(hi), upto = wave_scan_i(n);
  const int b = __builtin_popcountll(__ballot(upto <= s));
  const bool any = b < a.B;
  const int bs = any ? b : 0;
  return {bs, __builtin_amdgcn_readlane(upto - n, bs), hi, any, __builtin_amdgcn_readlane(gam, bs),
          __builtin_amdgcn_readlane(L, bs)};
}

// RING: tiles in flight per wave (see attention_kv4_plan). With one and two row
// blocks, 168 registers, three waves fit a SIMD; what is kept in scratch there is the
// merge's.
template <int D, int NQ, int RING, bool NT>
__global__ void __launch_bounds__(64 * kWaves, NQ == 1 || (NQ == 2 && RING == 1) ? 3 : 2)
attn_kv4_kernel(Kv4Args a) {
  constexpr int MQ = 16 * NQ;
  constexpr int DB = D / 16;
  constexpr int KS = D / 32;   // contraction steps of 32, dwords of codes per lane and row
  constexpr int EL = D / 4;    // elements per lane and row
  constexpr int kT = 64 * kWaves;
  using LL = Lds4<D, NQ>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[LL::kBytes];

  const int P = a.B * a.Hkv;
  const int window = a.window > 0 ? a.window : 0x7fffffff;
  const int sinks = a.sinks;
  int split, qc, g, b, gam, L, tiles_per = a.split_keys / kTile, n_splits = a.n_splits, pairs = P;
  size_t pair;  // with the splits of one, the record block of a split's partial: (pair n_splits + split)
  if (a.units > 0) {  // heads fastest, then units, then query chunks
    const int rest = (int)(blockIdx.x / (unsigned)a.Hkv);
    const Dealt d = deal(a, window, rest % a.units);
    if (!d.any) return;  // (the whole workgroup)
    g = (int)(blockIdx.x % (unsigned)a.Hkv);
    qc = rest / a.units;
    b = d.b, split = rest % a.units - d.first, gam = d.gam, L = d.L, tiles_per = d.tiles;
    n_splits = 1, pairs = a.Hkv * a.units, pair = (size_t)(g * a.units + d.first);
  } else {
    const int rest = (int)(blockIdx.x / (unsigned)P);
    const int code = a.order ? __builtin_amdgcn_readfirstlane(a.order[blockIdx.x])
                             : ((int)(blockIdx.x % (unsigned)P) * a.q_chunks + rest / n_splits) * n_splits +
                                   (n_splits - 1 - rest % n_splits);
    split = code % n_splits;
    qc = code / n_splits % a.q_chunks;
    const int pair_id = code / n_splits / a.q_chunks;
    g = pair_id % a.Hkv;
    b = pair_id / a.Hkv;
    gam = a.gamma[b];
    L = a.kv_len[b];
    pair = (size_t)pair_id;
  }
  const int job = (b * a.Hkv + g) * a.q_chunks + qc;
  const int G = a.Hq / a.Hkv;
  const int R = G * (a.gmax + 1);
  const bool valid = gam >= 0 && gam <= a.gmax && L >= gam + 1 && L <= a.L_cap;
  if (!valid && split == 0 && qc == 0 && g == 0 && threadIdx.x == 0 && a.status) {
    atomicOr(a.status, (gam < 0 || gam > a.gmax) ? SR_ST_GAMMA : SR_ST_KVLEN);
  }
  const int row0 = qc * MQ;
  const int row_end = min(R, row0 + MQ);
  const int Mb = valid ? G * (gam + 1) : 0;
  const int causal0 = valid ? L - gam - 1 : 0;  // cache position of new row 0
  const Reach<kTile> reach(causal0, valid ? L : 0, window, sinks);
  const int ns = (reach.tiles + tiles_per - 1) / tiles_per;  // splits that hold keys
  const bool work = row0 < Mb && split < ns;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int ws = wave_id();  // key stream
  const int l16 = lane & 15;
  const int lg = lane >> 4;

  // Four columns of output row r (bf16: rounded once, from the 32-bit sums).
  auto store = [&](int r, int col, const floatx4& x) __attribute__((always_inline)) {
    const int i = r / G, hh = g * G + r % G;
    const size_t at = ((size_t)(b * (a.gmax + 1) + i) * a.Hq + hh) * D + col;
    if (a.out_bf16) *(u32x2*)((uint16_t*)a.out + at) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    else *(floatx4*)((float*)a.out + at) = x;
  };
  if (!work) {
    // Split 0 of a query chunk without live rows (or of an invalid sequence) writes those rows as zero.
    if (split == 0)
      for (int idx = tid; idx < (row_end - row0) * (D / 4); idx += kT)
        store(row0 + idx / (D / 4), idx % (D / 4) * 4, floatx4{0.f, 0.f, 0.f, 0.f});
    return;
  }

  // slabs of (b, g) as buffer resources: 32-bit row offsets
  const size_t slab = ((size_t)b * a.Hkv + g) * (size_t)a.L_cap;
  const __amdgpu_buffer_rsrc_t rkc = make_rsrc(a.kc + slab * (D / 2), (size_t)a.L_cap * (D / 2));
  const __amdgpu_buffer_rsrc_t rvc = make_rsrc(a.vc + slab * (D / 2), (size_t)a.L_cap * (D / 2));
  const __amdgpu_buffer_rsrc_t rkp = make_rsrc(a.kp + slab * (D / 32), (size_t)a.L_cap * (D / 32));
  const __amdgpu_buffer_rsrc_t rvp = make_rsrc(a.vp + slab * (D / 32), (size_t)a.L_cap * (D / 32));
  const uint8_t* mrow = a.mask ? a.mask + (size_t)b * a.L_cap : nullptr;
  const __amdgpu_buffer_rsrc_t rm = make_rsrc(mrow ? mrow : a.kc, mrow ? (size_t)L : 0);  // (no mask: no traffic)

  floatx4 o[DB][NQ];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int qg = 0; qg < NQ; ++qg) {
    m_run[qg] = kNegInf;
    l_run[qg] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qg] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // The split's tiles [t0, t_end), dealt round-robin to the streams.
  const int t0 = split * tiles_per;
  const int t_end = min(reach.tiles, t0 + tiles_per);
  auto tile_key = [&](int t) __attribute__((always_inline)) { return t < t_end ? reach.start(t) : L; };
  constexpr int kPolicy = NT ? kStreamLoad : 0;
  // Every fetch issues the same loads; lanes past the length, and all lanes past
  // the stream's last tile, read out of range (as zero, with no traffic).
  const uint32_t lane_off = (uint32_t)(l16 * (D / 2) + lg * (EL / 2));
  const uint32_t lane_poff = (uint32_t)(l16 * (D / 32) + lg * EL / 32);
  auto fetch = [&](int t, Stage4<D>& st) __attribute__((always_inline)) {
    const int kb0 = tile_key(t);
    st.key = kb0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row0u = kb0 + u * 16;
      const bool in = l16 < L - row0u;
      const uint32_t off = in ? lane_off : kOutOfRange, poff = in ? lane_poff : kOutOfRange;
      const int at = row0u * (D / 2), pat = row0u * (D / 32);
      if constexpr (D == 128) {
        const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rkc, off, at, kPolicy));
        const u32x4 y = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rvc, off, at, kPolicy));
#pragma unroll
        for (int e = 0; e < 4; ++e) st.k[u][e] = x[e], st.v[u][e] = y[e];
      } else {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rkc, off, at, kPolicy));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rvc, off, at, kPolicy));
        st.k[u][0] = x[0], st.k[u][1] = x[1], st.v[u][0] = y[0], st.v[u][1] = y[1];
      }
      st.kp[u] = __builtin_amdgcn_raw_buffer_load_b8(rkp, poff, pat, kPolicy);
      st.vp[u] = __builtin_amdgcn_raw_buffer_load_b8(rvp, poff, pat, kPolicy);
    }
    st.mbyte = __builtin_amdgcn_raw_buffer_load_b8(rm, kb0 + (lane & (kTile - 1)), 0, 0);
  };
  // Tiles from key inner_lo to inner_hi are seen whole by every row (but for the mask).
  const int inner_lo = L - window, inner_hi = causal0 + 1 - kTile;
  // Bits 0 .. n - 1
  auto low_bits = [](int n) __attribute__((always_inline)) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };

  // This lane's part of the query rows: qf[qg][ks] holds Q[qg 16 + l16][lg EL + 8 ks ..].
  // (A third block's would not fit the registers beside its accumulators: its
  // rows are read from LDS, in the lanes' order, for every tile.)
  constexpr int kReg = LL::kReg;
  bf16x8 qf[kReg][KS];
#pragma unroll
  for (int qg = 0; qg < NQ; ++qg) {
    const int r = row0 + qg * 16 + l16;
    const int rc = min(r, Mb - 1), i = rc / G, hh = g * G + rc % G;
    const uint16_t* src = a.q + ((size_t)(b * (a.gmax + 1) + i) * a.Hq + hh) * D + lg * EL;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 y = *(const u32x4*)(src + ks * 8);
      const u32x4 x = r < Mb ? y : u32x4{0u, 0u, 0u, 0u};
      if (qg < kReg) qf[qg < kReg ? qg : 0][ks] = __builtin_bit_cast(bf16x8, x);
      else if (ws == 0) *(u32x4*)(lds + LL::kQ + (((qg - kReg) * KS + ks) * 64 + lane) * 16) = x;
    }
  }
  if (NQ > kReg) __syncthreads();
  auto query = [&](int qg, int ks) __attribute__((always_inline)) {
    return qg < kReg ? qf[qg < kReg ? qg : 0][ks]
                     : *(const bf16x8*)(lds + LL::kQ + (((qg - kReg) * KS + ks) * 64 + lane) * 16);
  };
  // This lane's V offsets in LDS: its row's first chunk as written, and the run it
  // names as read (the tile's other half is 16 rows on). The permutation turns the
  // low three bits of a chunk's number, so its other chunks lie at these offsets
  // with bits turned too, and columns 64 apart 128 bytes apart.
  const int v_write = ws * LL::kSlot + l16 * LL::kRow + chunk_at(lg * KS, l16) * 16;
  const int v_row = lg * 4 + (l16 >> 2);
  const int v_read = ws * LL::kSlot + v_row * LL::kRow + chunk_at((l16 & 3) >> 1, v_row) * 16 + (l16 & 1) * 8;

  // One tile for the first NL of the wave's row blocks (the others hold no live row).
  auto step = [&](auto blocks, int& t, Stage4<D>& st) __attribute__((always_inline)) {
    constexpr int NL = decltype(blocks)::value;
    const int kb0 = st.key;
    // keys that some row may see: below the length, in reach, valid
    const bool inner = kb0 >= inner_lo && kb0 <= inner_hi;
    uint32_t vbits = ~0u;
    if (rare(!inner)) vbits = low_bits(L - kb0) & (~low_bits(reach.first_key - kb0) | low_bits(sinks - kb0));
    if (mrow) vbits &= (uint32_t)__ballot(st.mbyte != 0u);
    if (rare(vbits != ~0u)) {  // V rows that no row sees are zeros, whatever they hold
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bool seen = (vbits >> (u * 16 + l16)) & 1u;
        st.vp[u] = seen ? st.vp[u] : (uint8_t)0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) st.v[u][ks] = seen ? st.v[u][ks] : 0u;
      }
    }
    // ---- S^T = K Q^T
    floatx4 sacc[2][NL];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) sacc[u][qg] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 ka[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        ka[u] = __builtin_bit_cast(bf16x8, widen(st.k[u][ks], __uint_as_float((uint32_t)st.kp[u] << 23)));
#pragma unroll
      for (int qg = 0; qg < NL; ++qg)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          sacc[u][qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[u], query(qg, ks), sacc[u][qg], 0, 0, 0);
    }
    // ---- V to LDS, while the products finish
    // (the offsets and the lane's numbers below are hidden from the optimiser, which
    // would keep all that follows from them in registers across the loop)
    int vw = v_write;
    asm volatile("" : "+v"(vw));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float scale = __uint_as_float((uint32_t)st.vp[u] << 23);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        *(u32x4*)(lds + (vw ^ (ks * 16)) + u * 16 * LL::kRow) = widen(st.v[u][ks], scale);
    }
    wave_lds_sync();
    t += RING * kWaves;
    __builtin_amdgcn_sched_barrier(0);
    fetch(t, st);
    __builtin_amdgcn_sched_barrier(0);
    // ---- online softmax, P in bf16 (lane: keys u 16 + lg 4 + e of query l16)
    if (rare(!inner || vbits != ~0u)) {  // (wave-uniform: not every row sees the whole tile)
      int r16 = l16, r4 = lg * 4;
      asm volatile("" : "+v"(r16), "+v"(r4));
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) {
        const int r = row0 + qg * 16 + r16;
        const int lim = r < Mb ? causal0 + r / G : -1;  // last key this query row sees
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int kl = (e / 4) * 16 + r4 + e % 4;
          const int k = kb0 + kl;
          const bool vis = (((vbits >> kl) & 1u) != 0u) & (k <= lim) & ((k > lim - window) | (k < sinks));
          sacc[e / 4][qg][e % 4] = vis ? sacc[e / 4][qg][e % 4] : kNegInf;
        }
      }
    }
    // A row's reference stands until a score exceeds it by more than 2^kLazy: only
    // then do its four lanes need their common maximum.
    bf16x8 pb[NL];
    float mt[NL];
    bool over = false;
#pragma unroll
    for (int qg = 0; qg < NL; ++qg) {
      mt[qg] = kNegInf;
#pragma unroll
      for (int e = 0; e < 8; ++e) mt[qg] = fmaxf(mt[qg], sacc[e / 4][qg][e % 4]);
      mt[qg] *= a.scale_log2;
      over |= mt[qg] > m_run[qg] + kLazy;
    }
    if (rare(__ballot(over) != 0ull)) {
#pragma unroll
      for (int qg = 0; qg < NL; ++qg) {
        const float m = max_across_rows(mt[qg]);
        const float mref = m > m_run[qg] + kLazy ? m : m_run[qg];
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
      float pk[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pk[e] = exp2_hw(fmaf(sacc[e / 4][qg][e % 4], a.scale_log2, -mr));
        l_run[qg] += pk[e];  // (of this lane's keys; the row's four lanes are summed at the end)
      }
      pb[qg] = __builtin_bit_cast(bf16x8, u32x4{to_bf16x2(pk[0], pk[1]), to_bf16x2(pk[2], pk[3]),
                                                to_bf16x2(pk[4], pk[5]), to_bf16x2(pk[6], pk[7])});
    }
    // ---- O^T += V^T P^T over the 32 keys: contraction slot lg 8 + e is key
    // lg 4 + e (e < 4) or 16 + lg 4 + e - 4, as the scores lie in the registers. Two
    // column blocks' reads are in flight before a block's products.
    int vr = v_read;
    asm volatile("" : "+v"(vr));
    shortx4 va[3][2];
    auto read = [&](int db) __attribute__((always_inline)) {
      const unsigned char* p0 = lds + (vr ^ (db % 4 * 32)) + db / 4 * 128;
      va[db % 3][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p0);
      va[db % 3][1] =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(p0 + 16 * LL::kRow));
    };
    read(0);
    read(1);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      if (db + 2 < DB) read(db + 2);
      const bf16x8 v =
          __builtin_bit_cast(bf16x8, __builtin_shufflevector(va[db % 3][0], va[db % 3][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int qg = 0; qg < NL; ++qg)
        o[db][qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[qg], o[db][qg], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    wave_lds_sync();  // this tile's LDS reads are issued before the slot is rewritten
  };

  __builtin_amdgcn_sched_barrier(0);
  Stage4<D> ring[RING];
  int tr[RING];
#pragma unroll
  for (int r = 0; r < RING; ++r) {
    tr[r] = t0 + ws + r * kWaves;
    fetch(tr[r], ring[r]);
    __builtin_amdgcn_sched_barrier(0);
  }
  // (a step past the stream's last tile reads nothing and adds nothing)
  auto loop = [&](auto blocks) __attribute__((always_inline)) {
    while (tr[0] < t_end) {
#pragma unroll
      for (int r = 0; r < RING; ++r) step(blocks, tr[r], ring[r]);
    }
  };
  const int live = min(NQ, (Mb - row0 + 15) / 16);
  if (NQ >= 3 && live >= 3) loop(std::integral_constant<int, NQ >= 3 ? 3 : 1>{});
  else if (NQ >= 2 && live >= 2) loop(std::integral_constant<int, NQ >= 2 ? 2 : 1>{});
  else loop(std::integral_constant<int, 1>{});
#pragma unroll
  for (int qg = 0; qg < NQ; ++qg) l_run[qg] = sum_across_rows(l_run[qg]);
  __syncthreads();

  const JobRows J{row0, row_end, Mb, R, split, ns, n_splits, job, pairs, pair};
  merge_and_store<typename LL::Merge, D, NQ, 1, LL::kBytes, true>(lds, o, m_run, l_run, J, a.part_o, a.part_ml, a.counters, store);
}

typedef void (*Kv4Kernel)(Kv4Args);

// (more than one query chunk takes at least two row blocks)
template <int D>
Kv4Kernel pick_kv4(int nq, int ring, bool nt) {
  if (nq == 1) return attn_kv4_kernel<D, 1, 2, true>;
  if (nq == 3) return nt ? attn_kv4_kernel<D, 3, 1, true> : attn_kv4_kernel<D, 3, 1, false>;
  if (ring == 1) return nt ? attn_kv4_kernel<D, 2, 1, true> : attn_kv4_kernel<D, 2, 1, false>;
  return nt ? attn_kv4_kernel<D, 2, 2, true> : attn_kv4_kernel<D, 2, 2, false>;
}
Kv4Kernel pick_kv4(int D, int nq, int ring, int q_chunks) {
  return D == 64 ? pick_kv4<64>(nq, ring, q_chunks == 1) : pick_kv4<128>(nq, ring, q_chunks == 1);
}

}  // namespace

int attention_kv4_plan(int B, int gamma_max, int Hq, int Hkv, int D, int cache_rows, int window, int sinks,
                       AttentionPlan* plan) {
  const int L = reach_cap(kTile, gamma_max, cache_rows, window, sinks);  // keys of a sequence at most
  const int R = Hq / Hkv * (gamma_max + 1);
  plan->qg = 1;
  plan->q_chunks = (R + 16 * kMaxNQ4 - 1) / (16 * kMaxNQ4);
  plan->nq = ((R + plan->q_chunks - 1) / plan->q_chunks + 15) / 16;
  const int cus = device_cu_count();
  if (cus <= 0) return SR_ELAUNCH;
  const long pairs = (long)B * Hkv * plan->q_chunks;
  // Splits: the count whose time is least, in units of a key's time in a workgroup
  // (two workgroups on a CU take little longer than one): the keys of a split,
  // times the workgroups over two per CU, plus the merge of each split's partial.
  // (32/8 heads of 128, gamma 5: one sequence of 32768 keys 230 us with 1 split, 26
  // with 24, 31 with 48; 24 sequences of 256 to 8192 keys 65 with 1, 41 with 3 or 4, 50
  // with 10; 16 sequences of 2048 24 with 1, 20 with 2 to 4, 33 with 8.)
  constexpr long kPerSplit = 64;
  // A window shorter than the cache makes the sequences alike, so that nothing
  // balances a second turn of workgroups (46 sequences of 1648 positions, 4/1 heads by 8,
  // gamma 4: 34 us with one split, 45 with two).
  const bool alike = L < cache_rows;
  const long most = (2L * cus + pairs - 1) / pairs;
  long splits = 1, best = 0;
  for (long n = 1; n <= most; ++n) {
    const long keys = (L + n - 1) / n, jobs = pairs * n;
    const long t = (jobs <= 2L * cus ? keys : alike ? (jobs + 2L * cus - 1) / (2L * cus) * keys : keys * jobs / (2L * cus)) +
                   (n > 1 ? n * kPerSplit : 0);
    if (n == 1 || t < best) best = t, splits = n;
  }
  const long max_splits = (L + kTile - 1) / kTile;
  if (splits > max_splits) splits = max_splits;
  // Offsets into the partial arrays are 32-bit (buffer addressing): below 2^31 bytes.
  const long max_by_offset = 0x7fffffffL / ((long)D * 4 * B * Hkv * R);
  if (splits > max_by_offset) splits = max_by_offset > 1 ? max_by_offset : 1;
  int sk = (int)((L + splits - 1) / splits);
  sk = (sk + kTile - 1) / kTile * kTile;
  plan->split_keys = sk;
  plan->n_splits = (L + sk - 1) / sk;
  plan->follow = 0;
  // Tiles in flight per wave: two, but one with three row blocks, whose accumulators
  // leave no registers for a second without keeping others in scratch (16 sequences of
  // 2048 keys, 32/8 heads of 128, gamma 8: 22 us with one, 26 with two; 256 of 4096: 270
  // and 287), and one with two row blocks and more than four workgroups per CU, for a
  // third wave per SIMD (256 sequences of 2048 keys, gamma 5: 121 and 135; 24 ragged ones,
  // 2.25 workgroups per CU: 46 and 39).
  // Up to 64 sequences on no more workgroups than CUs: the kernel deals them by the
  // lengths, which the host does not know, to two workgroups per CU (32/8 heads of 128,
  // gamma 5, us with the splits above and dealt: 18 sequences of 4456 keys 39 and 28, 12 of
  // 256 to 8192 30 and 27, 24 of 256 to 8192 39 and 37, one of 512 10.8 and 11.3). With more, a
  // ragged batch has few splits to give away: 46 sequences of 1292 to 15505 89 and 111.
  plan->units = 0;
  if (B <= kMaxDealt && pairs <= cus && L > 4 * kMergeKeys) {
    const int tiles = (L + kTile - 1) / kTile, least = least_tiles(tiles);
    const long room = 2L * cus / (Hkv * plan->q_chunks), need = (long)B * ((tiles + least - 1) / least);
    plan->units = (int)(need < room ? need : room);
    plan->n_splits = (plan->units + B - 1) / B;
  }
  const long n_jobs = plan->units > 0 ? (long)plan->units * Hkv * plan->q_chunks : (long)plan->n_splits * pairs;
  plan->ring = plan->nq == 3 || (plan->nq == 2 && n_jobs > 4L * cus) ? 1 : 2;
  const long target =
      (long)cus * resident_per_cu((const void*)pick_kv4(D, plan->nq, plan->ring, plan->q_chunks), 64 * kWaves, 0);
  // [arrival counters, one per 128-byte line][partial o][partial (m, l)][order]
  const size_t counters = (size_t)pairs * kCounterStride * sizeof(uint32_t);
  plan->part_offset = counters;
  const size_t records = plan->units > 0 ? (size_t)Hkv * plan->units : (size_t)B * Hkv * plan->n_splits;
  size_t bytes = plan->units > 0 || plan->n_splits > 1 ? counters + records * R * (D + 2) * sizeof(float) : 0;
  // (Up to 1024 keys what it balances is less than the order kernel's 5 us: 256
  // sequences of 100 to 300 keys 36.6 us with it, 34.1 without, of 100 to 700 45.3 and 43.6.)
  plan->ordered = n_jobs > target && L > 1024 && plan->units == 0 ? 1 : 0;
  plan->order_offset = (bytes + 15) / 16 * 16;
  if (plan->ordered) bytes = plan->order_offset + (size_t)n_jobs * sizeof(int32_t);
  plan->workspace_bytes = bytes;
  return SR_OK;
}

int launch_attention_kv4(const void* q, const void* k_codes, const void* k_powers, const void* v_codes,
                         const void* v_powers, const uint8_t* cache_mask, const int32_t* kv_len, const int32_t* gamma,
                         void* out, bool out_bf16, int B, int gamma_max, int Hq, int Hkv, int D, int L_cap, int window,
                         int sinks, float scale, void* workspace, const AttentionPlan& plan, int32_t* status,
                         hipStream_t stream) {
  const int R = Hq / Hkv * (gamma_max + 1);
  float* part_o = workspace ? (float*)((char*)workspace + plan.part_offset) : nullptr;
  const size_t records = plan.units > 0 ? (size_t)Hkv * plan.units : (size_t)B * Hkv * plan.n_splits;
  float* part_ml = part_o ? part_o + records * R * D : nullptr;
  int32_t* order = plan.ordered ? (int32_t*)((char*)workspace + plan.order_offset) : nullptr;
  if (order && launch_attention_order(kv_len, gamma, B, gamma_max, Hkv, plan.q_chunks, L_cap, window, sinks, kTile,
                                      plan.split_keys, plan.n_splits, order, stream) != SR_OK)
    return SR_ELAUNCH;
  const Kv4Args a{(const uint16_t*)q, (const uint8_t*)k_codes, (const uint8_t*)k_powers, (const uint8_t*)v_codes,
                  (const uint8_t*)v_powers, cache_mask, kv_len, gamma, out, out_bf16, part_o, part_ml,
                  (uint32_t*)workspace, order, B, gamma_max, Hq, Hkv, L_cap, window, sinks, scale * kLog2e,
                  plan.split_keys, plan.n_splits, plan.q_chunks, plan.units, status};
  const dim3 grid((unsigned)((plan.units > 0 ? (long)plan.units : (long)plan.n_splits * B) * plan.q_chunks * Hkv));
  hipLaunchKernelGGL(pick_kv4(D, plan.nq, plan.ring, plan.q_chunks), grid, dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
}

}  // namespace sr
