// Verification attention over a bf16 cache, without and with a window: the dispatch
// order of ragged batches, the launch plan and the launches. The kernel is in
// attention_split.h; its forms with a window are compiled in attention_window.hip.

#include "attention_split.h"

namespace sr {
namespace {

// The dispatch order of the split workgroups when there are more than fit on
// the device at once (one workgroup of kOrderThreads): every job (sequence,
// kv head, query chunk, split) by decreasing key count (in 16-key tiles, a
// counting sort), empty jobs last, so that the workgroups that start last
// are the shortest and the device does not idle behind a few long ones.
// Jobs of equal count take any order among themselves (the results do not
// depend on the order). Entry: ((b Hkv + g) q_chunks + qc) n_splits + split;
// the jobs of one (sequence, split) are consecutive, kv head fastest.
constexpr int kOrderThreads = 1024;
constexpr int kOrderBuckets = 1024;  // 0: empty; t: t tiles (the last bucket also takes longer jobs)
constexpr int kOrderKept = 4;        // buckets a thread keeps between the two passes
static_assert(kOrderThreads == kOrderBuckets, "one scan element per thread");
__global__ void __launch_bounds__(kOrderThreads)
attn_order_kernel(const int32_t* __restrict__ kv_len, const int32_t* __restrict__ gamma, int B, int gmax,
                  int Hkv, int q_chunks, int L_cap, int window, int sinks, int tile, int split_keys, int n_splits,
                  int32_t* __restrict__ order) {
  __shared__ int cnt[kOrderBuckets];
  __shared__ int wsum[kOrderThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per_item = Hkv * q_chunks;  // jobs of one (sequence, split)
  const int n_items = B * n_splits;
  auto bucket = [&](int item) __attribute__((always_inline)) {
    const int b = item / n_splits, sp = item % n_splits;
    const int gam = gamma[b], L = kv_len[b];
    const bool valid = gam >= 0 && gam <= gmax && L >= gam + 1 && L <= L_cap;
    int keys = L;  // with a window, the keys of the tiles in reach
    if (window > 0 && valid) {
      if (tile == 16) keys = Reach<16>(L - gam - 1, L, window, sinks).tiles * 16;
      else keys = Reach<32>(L - gam - 1, L, window, sinks).tiles * 32;
    }
    const int len = valid ? min(keys, (sp + 1) * split_keys) - sp * split_keys : 0;
    return len <= 0 ? 0 : min((len + kWaveKeys - 1) / kWaveKeys, kOrderBuckets - 1);
  };
  cnt[tid] = 0;
  __syncthreads();
  // the first kOrderKept items of a thread keep their bucket for the second pass
  int kept[kOrderKept];
#pragma unroll
  for (int u = 0; u < kOrderKept; ++u) {
    const int item = tid + u * kOrderThreads;
    kept[u] = item < n_items ? bucket(item) : 0;
    if (item < n_items) atomicAdd(&cnt[kept[u]], per_item);
  }
  for (int item = tid + kOrderKept * kOrderThreads; item < n_items; item += kOrderThreads)
    atomicAdd(&cnt[bucket(item)], per_item);
  __syncthreads();
  // start of bucket t: the jobs of every longer bucket (thread t holds
  // bucket kOrderBuckets - 1 - t, an inclusive scan in thread order)
  const int t_b = kOrderBuckets - 1 - tid;
  const int c = cnt[t_b];
  int incl = c;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(incl, d, 64);
    if (lane >= d) incl += o;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  for (int i = 0; i < w; ++i) incl += wsum[i];
  cnt[t_b] = incl - c;  // now each bucket's next free position (each thread rewrites only its own)
  __syncthreads();
  auto place = [&](int item, int bk) __attribute__((always_inline)) {
    const int pos = atomicAdd(&cnt[bk], per_item);
    const int b = item / n_splits, sp = item % n_splits;
    for (int j = 0; j < per_item; ++j) {
      // kv head fastest: with a multiple of 8 heads the query chunks of one
      // (pair, split) fall on one XCD and share its L2
      const int qc = j / Hkv, g = j % Hkv;
      order[pos + j] = ((b * Hkv + g) * q_chunks + qc) * n_splits + sp;
    }
  };
#pragma unroll
  for (int u = 0; u < kOrderKept; ++u) {
    const int item = tid + u * kOrderThreads;
    if (item < n_items) place(item, kept[u]);
  }
  for (int item = tid + kOrderKept * kOrderThreads; item < n_items; item += kOrderThreads) place(item, bucket(item));
}

SplitKernel pick_split(int D, int nq, int qg, int q_chunks, bool follow) {
  if (follow) return D == 64 ? pick_split<64, true, false>(nq, qg, q_chunks) : pick_split<128, true, false>(nq, qg, q_chunks);
  return D == 64 ? pick_split<64, false, false>(nq, qg, q_chunks) : pick_split<128, false, false>(nq, qg, q_chunks);
}

}  // namespace

int attention_plan(int B, int gamma_max, int Hq, int Hkv, int D, int cache_rows, int window, int sinks,
                   AttentionPlan* plan) {
  const int L_cap = reach_cap(kWaveKeys, gamma_max, cache_rows, window, sinks);  // keys of a sequence at most
  const int G = Hq / Hkv;
  const int R = G * (gamma_max + 1);
  // Up to 48 rows: one four-wave group of ceil(R / 16) row blocks. Beyond:
  // two groups of two (up to 64 rows) or three blocks, in as many query
  // chunks of 96 rows as needed.
  if (R <= 16 * kMaxNQ) {
    plan->qg = 1;
    plan->nq = (R + 15) / 16;
  } else {
    plan->qg = kMaxQG;
    plan->nq = R <= 2 * 32 ? 2 : kMaxNQ;
  }
  const int rows_per_chunk = 16 * plan->nq * plan->qg;
  plan->q_chunks = (R + rows_per_chunk - 1) / rows_per_chunk;
  const int cus = device_cu_count();
  if (cus <= 0) return SR_ELAUNCH;
  // With a window, more than 48 rows go to chunks of up to 48, four waves each, which
  // read the same keys through an L2 but fit two to a CU and waste fewer row
  // blocks; two groups in eight waves stay where they leave no CU idle, save no rows
  // and stream long. (64 query heads on 8 of 128, us in eight waves and in chunks: one sequence
  // of 1024 positions, 64 rows, 20.0 and 13.6; 16 of 1024 28.8 and 23.4, of 3000
  // 45.5 and 53.7; 32 of 512 25.2 and 24.3, of 640 26.6 and 29.9; 40 of 2048,
  // 72 rows, 118 and 98, 136 rows 164 and 120; 256 of 512, 72 rows, 217 and 176.
  // Where the jobs divide the CUs, by the keys of a CU, jobs L_cap / 256, over 1 to 32 sequences,
  // both dimensions, 56 to 192 rows: 256 keys 29 and 23, 512 33 and 31, 750 37 and 38, 1024
  // 47 and 49, 2048 70 and 82 for 96 rows of 128, at 64 about the same from 400 on. Rows that
  // chunks save blocks of, 112 of 128 in three, are faster at every length, 136 and 144 up to
  // 2048 and within 8% beyond; of 64 those lose up to a fifth from 1024 on.)
  bool chunked = false;
  if (window > 0 && plan->qg > 1) {
    const int chunks = (R + 16 * kMaxNQ - 1) / (16 * kMaxNQ);
    const long jobs = (long)B * Hkv * plan->q_chunks;
    const bool even = jobs <= cus && cus % jobs == 0;
    if (!even || chunks < kMaxQG * plan->q_chunks || jobs * L_cap <= 600l * cus) {
      chunked = true;
      plan->qg = 1;
      plan->q_chunks = chunks;
      plan->nq = ((R + chunks - 1) / chunks + 15) / 16;
    }
  }
  const int threads = plan->qg == 1 ? Shape<1>::kThreads : Shape<kMaxQG>::kThreads;
  const int per_cu = resident_per_cu((const void*)(window > 0 ? window_kernel(D, plan->nq, plan->qg, plan->q_chunks, false)
                                                                 : pick_split(D, plan->nq, plan->qg, plan->q_chunks, false)), threads, 0);
  const long pairs = (long)B * Hkv * plan->q_chunks;
  const long target = (long)cus * per_cu;
  // Splits: the count, up to one workgroup per CU, whose time is least for
  // sequences of L_cap keys each. In units of a key's time in a workgroup (16 ns
  // at D = 128, a CU's share of HBM): the keys of a split, times the workgroups
  // the busiest CU gets, and the merge of each split's partial, 0.2 to 0.35 us
  // or about 16 keys. One sequence of 2048 keys, 32/8 heads of 128, gamma 5:
  // 24.8 us with the 32 splits that fill the CUs and the merge of before, 18.8
  // with the present merge, 16.6 with 11.
  const long most = ((long)cus + pairs - 1) / pairs;
  constexpr long kPerSplit = 16;
  // With two query groups a softmax reference serves up to two tiles of a wave, so
  // where one workgroup per CU leaves a wave one tile (64 keys per split), the
  // splits stay that short (see follow below).
  constexpr long kTileKeys = kWaves * kWaveKeys;
  const long least = plan->qg == 1 || L_cap > most * kTileKeys ? 1 : (L_cap + kTileKeys - 1) / kTileKeys;
  long splits = least, best = 0;
  for (long n = least; n <= most; ++n) {
    const long t = (pairs * n + cus - 1) / cus * ((L_cap + n - 1) / n) + (n > 1 ? n * kPerSplit : 0);
    if (n == least || t < best) {
      best = t;
      splits = n;
    }
  }
  const bool few = splits < most;
  // Lengths are not known here and may be anything up to L_cap. Where the pairs
  // go into the CUs a few times with a remainder, that count is one workgroup
  // per CU or fewer, and a ragged batch waits for its longest sequence alone on
  // its CU. Two workgroups per CU instead (on long caches, where a merge is
  // little, as many as fit), but for caches so short that the merge costs more
  // than the balance gives, the more so where one split each leaves few CUs idle.
  // (32/8 heads of 128, 256 to 8192 keys: 12 sequences 101 us with 2 splits, 58
  // with 5; 17: 133 with 1, 75 with 3; 24: 170 with 1, 114 with 2. 2048 keys each:
  // 17: 41.4 and 33.6; 24: 41.6 and 44.7; 31: 43 and 50. 512 keys each, 24: 11 and
  // 12.) A single row block has fewer products per key and is near HBM's rate with
  // fewer CUs; two query groups take a CU each, so their second workgroup only
  // waits its turn, which pays with few splits of long caches.
  const long whole = pairs < cus ? cus / pairs : 0;
  if (whole >= 1 && cus % pairs != 0) {
    const long busy = 10 * pairs * whole / cus;  // tenths of the CUs, the pairs taken a whole number of times
    if (plan->qg == 1 && whole <= 7) {
      const bool idle = whole > 1 || busy < (plan->nq > 1 ? 8 : 7);
      if (L_cap >= 6000 && (plan->nq > 1 || !idle)) splits = target / pairs;
      else if (L_cap >= 1000 && idle) splits = 2 * cus / pairs;
    } else if (plan->qg > 1 && whole <= 2 && L_cap >= (busy < 6 ? 1500 : 3000)) {
      splits = 2 * cus / pairs;
    }
  }
  // Bound a workgroup's keys, so the last workgroups of a ragged batch do not
  // run long after the rest have finished.
  const long by_length = (L_cap + kMaxSplitKeys - 1) / kMaxSplitKeys;
  if (splits < by_length) splits = by_length;
  const long max_splits = (L_cap + kWaveKeys - 1) / kWaveKeys;
  if (splits < 1) splits = 1;
  if (splits > max_splits) splits = max_splits;
  // Offsets into the partial arrays are 32-bit (buffer addressing): keep
  // them below 2^31 bytes.
  const long rec_per_split = (long)B * Hkv * R;
  const long max_by_offset = (long)(0x7fffffffL / ((long)D * 4 * (rec_per_split > 0 ? rec_per_split : 1)));
  if (splits > max_by_offset) splits = max_by_offset > 1 ? max_by_offset : 1;
  int sk = (int)((L_cap + splits - 1) / splits);
  sk = (sk + kWaveKeys - 1) / kWaveKeys * kWaveKeys;
  plan->split_keys = sk;
  plan->n_splits = (L_cap + sk - 1) / sk;
  // The key that a reference was taken from has P = 1, without rounding: one per
  // wave with a lazy reference. Fewer and longer splits would have fewer of
  // them (64 to 8192 normal keys: 1.05e-3 off the 64-bit result with one tile
  // per wave, 1.5e-3 with three), so there the reference follows the tiles
  // (one such key per tile whatever the length: 1.05e-3 again). With a window that costs
  // a call 3 to 10% (one sequence of 8192 positions, 72 rows, 25.4 and 26.6 us), so there a
  // wave of one tile, whose reference is that tile's maximum either way, stays lazy.
  plan->follow = few && (window == 0 || plan->split_keys > kTileKeys) ? 1 : 0;
  // Rows in chunks with a window are as exact as the two groups without one: where those
  // follow, or leave a wave one tile, a wave of several tiles follows here. (2 sequences
  // of 2048 keys, 72 rows: 1.52e-3 off where the reference is lazy, 1.01e-3 where it follows.)
  if (chunked && plan->split_keys > kTileKeys) {
    AttentionPlan groups;
    const int rc = attention_plan(B, gamma_max, Hq, Hkv, D, L_cap, 0, 0, &groups);
    if (rc != SR_OK) return rc;
    plan->follow = groups.follow || groups.split_keys <= kTileKeys ? 1 : 0;
  }
  // [arrival counters: B*Hkv*q_chunks, one per 128-byte line][partial o][partial (m, l)][order]
  const size_t counters = (size_t)B * Hkv * plan->q_chunks * kCounterStride * sizeof(uint32_t);
  plan->part_offset = counters;
  size_t bytes = plan->n_splits > 1 ? counters + (size_t)B * Hkv * plan->n_splits * R * (D + 2) * sizeof(float) : 0;
  const long n_jobs = (long)plan->n_splits * pairs;
  // With a window, sequences differ by its length at most, and for short ones that is less
  // than the order kernel's 5 us and the table's reads. With one or two query chunks it is
  // up to 704 keys, whatever the number of jobs (33 to 256 sequences of half to three
  // windows, or of up to one; us without and with the order: 32/32 heads of 64, 33 sequences
  // of 256 positions 16.1 and 20.6, 256 of 704 259 and 254; 64/8 of 128, gamma 8, 128 of
  // 512 85 and 92, 256 of 704 207 and 205, and of 2 to 512 97 and 123). From three chunks on
  // the order also brings a pair's chunks together, which then share its keys in an
  // L2 (64/8 of 128, gamma 16, 256 sequences of 256 150 and 137, of 704 299 and 220), so it
  // goes only up to 128 keys, or for a few chunks more than fit at once (24 of 512 27 and 31).
  const bool alike = window > 0 && (L_cap <= 2 * kTileKeys ||
                                    (L_cap <= 704 && (plan->q_chunks <= 2 || 2 * n_jobs <= 3 * target)));
  plan->ordered = n_jobs > target && !alike ? 1 : 0;
  plan->order_offset = (bytes + 15) / 16 * 16;
  if (plan->ordered) bytes = plan->order_offset + (size_t)n_jobs * sizeof(int32_t);
  plan->workspace_bytes = bytes;
  return SR_OK;
}

int launch_attention_order(const int32_t* kv_len, const int32_t* gamma, int B, int gamma_max, int Hkv, int q_chunks,
                           int L_cap, int window, int sinks, int tile, int split_keys, int n_splits, int32_t* order,
                           hipStream_t stream) {
  hipLaunchKernelGGL(attn_order_kernel, dim3(1), dim3(kOrderThreads), 0, stream, kv_len, gamma, B, gamma_max, Hkv,
                     q_chunks, L_cap, window, sinks, tile, split_keys, n_splits, order);
  return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
}

int launch_verify_attention(const void* q, const void* k_cache, const void* v_cache,
                            const uint8_t* cache_mask, const int32_t* kv_len,
                            const int32_t* gamma, void* out, bool out_bf16, int B, int gamma_max, int Hq,
                            int Hkv, int D, int L_cap, int window, int sinks, float scale, void* workspace,
                            const AttentionPlan& plan, int32_t* status, hipStream_t stream) {
  const int G = Hq / Hkv;
  const int R = G * (gamma_max + 1);
  uint32_t* counters = (uint32_t*)workspace;
  float* part_o = workspace ? (float*)((char*)workspace + plan.part_offset) : nullptr;
  float* part_ml = part_o ? part_o + (size_t)B * Hkv * plan.n_splits * R * D : nullptr;
  dim3 grid((unsigned)((long)plan.n_splits * plan.q_chunks * B * Hkv));
  const int threads = plan.qg == 1 ? Shape<1>::kThreads : Shape<kMaxQG>::kThreads;
  int32_t* order = plan.ordered ? (int32_t*)((char*)workspace + plan.order_offset) : nullptr;
  if (order && launch_attention_order(kv_len, gamma, B, gamma_max, Hkv, plan.q_chunks, L_cap, window, sinks, kWaveKeys,
                                      plan.split_keys, plan.n_splits, order, stream) != SR_OK)
    return SR_ELAUNCH;
  const SplitKernel kernel = window > 0 ? window_kernel(D, plan.nq, plan.qg, plan.q_chunks, plan.follow != 0)
                                        : pick_split(D, plan.nq, plan.qg, plan.q_chunks, plan.follow != 0);
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, (const uint16_t*)q, (const uint16_t*)k_cache,
                     (const uint16_t*)v_cache, cache_mask, kv_len, gamma, out, out_bf16, part_o, part_ml, counters,
                     order, B, gamma_max, Hq, Hkv, L_cap, window, sinks, scale * kLog2e, plan.split_keys, plan.n_splits,
                     plan.q_chunks, status);
  return hipGetLastError() == hipSuccess ? SR_OK : SR_ELAUNCH;
}

}  // namespace sr
