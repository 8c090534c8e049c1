// What a kernel that reads and writes every value once leaves in the caches.
//
// The L2s of the eight XCDs hold 32 MiB together. While a call's inputs and
// outputs fit, the outputs stay there for the kernel that reads them next
// (kKeep). Where they do not, the inputs, which nothing reads again, are marked
// to be dropped first, so that they do not drive the outputs out (kReadOnce);
// and beyond what the memory-side cache keeps for the reader as well, the outputs are
// marked too (kPass). Normalised and rotated heads, alone / followed by a
// copy of the result, us (four steps a wave):
//    16 MB   keep  7.4 / 12.5   read once  7.7 / 12.9   pass  6.2 / 13.0
//    42 MB        12.3 / 23.2             12.4 / 20.8         9.8 / 21.3
//    86 MB        24.0 / 39.6             21.5 / 36.6        19.8 / 40.6
//   333 MB        69.1 / 139              65.1 / 124         58.8 / 126
//   1.2 GB         207 / 438               206 / 443          190 / 425
// Rows appended in 4 bits, with the values that attention will see:
//    38 MB        11.2 / 21.4             13.2 / 20.6        12.8 / 22.4
//    76 MB        23.0 / 34.2             19.6 / 32.1        19.4 / 36.8
//   228 MB        50.2 / 107              50.1 / 101         44.1 / 101
#pragma once

#include "sr_internal.h"

namespace sr {

enum Caching { kKeep, kReadOnce, kPass };

// of a call that moves at most this many bytes in and out
inline Caching caching_of(long bytes) {
  return bytes < (36l << 20) ? kKeep : bytes < (128l << 20) ? kReadOnce : kPass;
}

template <int CACHING>
__device__ __forceinline__ u32x4 load_once(const uint16_t* p) {
  if constexpr (CACHING == kKeep) return *(const u32x4*)p;
  else return __builtin_nontemporal_load((const u32x4*)p);
}
template <int CACHING>
__device__ __forceinline__ void store_once(uint16_t* p, u32x4 v) {
  if constexpr (CACHING == kPass) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

}  // namespace sr
