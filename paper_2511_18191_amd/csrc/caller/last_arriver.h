// Work split over workgroups and finished in the same launch by the one that comes last, without memory that was cleared beforehand.
//
// Every workgroup of a group leaves its part in the workspace and then its tag, a word that no other call uses, in its own slot.  It
// then looks at the group's slots: whoever finds all tags there finishes.  A tag is there before its workgroup looks, so the one whose
// tag came last finds them all; two that came together may both, and then do the same work twice, to the same values.  Nobody waits.
// The finisher clears the slots: a replayed graph brings the same tag again.
// Parts, tags and looks go past the XCDs' own caches (relaxed, agent scope), in the order of the waits between them: fences, which write a whole L2
// back, queued up here (64 rows of 131072 fp32 probabilities, 32 workgroups a row: 244 us instead of 20).
#pragma once
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "tsd_internal.h"

namespace tsd {

// A tag that the memory does not hold by chance: calls are counted, and the count is spread over 64 bits.
inline uint64_t new_tag() {
  static std::atomic<uint64_t> calls{0};
  const uint64_t tag = (calls.fetch_add(1, std::memory_order_relaxed) + 1) * 0x9E3779B97F4A7C15ull;  // (odd: no two calls have the same)
  return tag ? tag : 1;
}

#if defined(__HIPCC__)
// (V: 4 or 8 bytes)
template <typename V>
using WordOf = std::conditional_t<sizeof(V) == 8, uint64_t, uint32_t>;
template <typename V>
__device__ __forceinline__ void leave(V* to, V v) {
  __hip_atomic_store(reinterpret_cast<WordOf<V>*>(to), __builtin_bit_cast(WordOf<V>, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename V>
__device__ __forceinline__ V left(const V* from) {
  return __builtin_bit_cast(V, __hip_atomic_load(reinterpret_cast<const WordOf<V>*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// For a whole workgroup, once it has left its part: whether it finishes the group of `n`, whose slot `own` is its.
__device__ __forceinline__ bool came_last(uint64_t* slots, int n, int own, uint64_t tag) {
  __shared__ int last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every wavefront's part is there
  __syncthreads();
  if (threadIdx.x < 64) {
    if (threadIdx.x == 0) __hip_atomic_exchange(slots + own, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // ... and the tag
    bool all = true;
    for (int i = threadIdx.x; i < n; i += 64) all &= __hip_atomic_load(slots + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == tag;
    all = __all(all);
    if (threadIdx.x == 0) last = all;
  }
  __syncthreads();
  return last;
}

// By the finisher, at its end.
__device__ __forceinline__ void clear_slots(uint64_t* slots, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) __hip_atomic_store(slots + i, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
#endif

}  // namespace tsd
