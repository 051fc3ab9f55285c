// A draw from a row of weights, p or what p has over q: the first v with w_0 + .. + w_v > u W, W the sum of all, in 64 bits.
//
// A row goes in segments of kSegment elements, summed by a wavefront each; then the segment that crosses u W is found, and the token inside
// it.  Rows start anywhere (an odd vocabulary), so 16-byte loads need no alignment beyond the element's.
#pragma once
#include "last_arriver.h"

namespace tsd {

constexpr int kSegment = 1024;
constexpr int kNoToken = -1;

#if defined(__HIPCC__)
__device__ __forceinline__ long token_at(const void* p, long i, int wide) {
  return wide ? reinterpret_cast<const long*>(p)[i] : (long)reinterpret_cast<const int*>(p)[i];
}

// The weights of a draw: p, or what p has over q (a certain draft's q is 1 at its token).
template <typename T>
struct Weights {
  const T* p;
  const T* q;      // NULL: p alone
  int without;     // this token has none (kNoToken: every token has its own)
  // Compared in 32 bits, subtracted in 64; what is no finite positive number weighs nothing.
  __device__ __forceinline__ double of(float x, float y, long v) const {
    const bool some = x > y && x < INFINITY && y > -INFINITY && (v == kNoToken || (int)v != without);
    return (double)(some ? x : 0.f) - (double)(some ? y : 0.f);
  }
};

// 16 bytes of a row, which may start at any element.  In words: as elements, the compiler unpacks each load where it is issued, and waits for it.
typedef unsigned Words __attribute__((ext_vector_type(4)));
template <typename T>
struct alignas(sizeof(T)) Pack {
  unsigned char bytes[16];
};
template <typename T>
__device__ __forceinline__ Words load_pack(const T* from) {
  return __builtin_bit_cast(Words, *reinterpret_cast<const Pack<T>*>(from));
}
template <typename T>
__device__ __forceinline__ float element(const Words& w, int j) {
  if constexpr (sizeof(T) == 4)
    return __uint_as_float(w[j]);
  else
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);  // (bf16 is the upper half of an fp32)
}

// C packs of weights, pack c from element v0 + c * STEP on; 0 beyond V.  inside: all of them lie in the row (the same in every lane).
template <typename T, int C, int STEP>
__device__ __forceinline__ void load_weights(const Weights<T>& w, long v0, int V, bool inside, double (&d)[C * (16 / sizeof(T))]) {
  constexpr int E = 16 / sizeof(T);
  if (inside) {
    Words x[C];
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = load_pack(w.p + v0 + c * STEP);
    if (w.q) {
      Words y[C];
#pragma unroll
      for (int c = 0; c < C; ++c) y[c] = load_pack(w.q + v0 + c * STEP);
#pragma unroll
      for (int i = 0; i < C * E; ++i) d[i] = w.of(element<T>(x[i / E], i % E), element<T>(y[i / E], i % E), kNoToken);
    } else {
#pragma unroll
      for (int i = 0; i < C * E; ++i) d[i] = w.of(element<T>(x[i / E], i % E), 0.f, v0 + i / E * STEP + i % E);
    }
  } else {
#pragma unroll
    for (int i = 0; i < C * E; ++i) {
      const long v = v0 + i / E * STEP + i % E;
      d[i] = 0.0;
      if (v < V) d[i] = w.of((float)w.p[v], w.q ? (float)w.q[v] : 0.f, v);
    }
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

// Sum of segment s (by one wavefront): a lane's packs lie 64 packs apart.
template <typename T>
__device__ __forceinline__ double segment_sum(const Weights<T>& w, long s, int V) {
  constexpr int E = 16 / sizeof(T), C = kSegment / (64 * E);
  double d[C * E], sum = 0.0;
  load_weights<T, C, 64 * E>(w, s * kSegment + (threadIdx.x & 63) * E, V, (s + 1) * kSegment <= V, d);
#pragma unroll
  for (int j = 0; j < C * E; ++j) sum += d[j];
  return wave_sum(sum);
}

// Inclusive sums over the wavefront's lanes.
__device__ __forceinline__ double wave_scan(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// The first segment whose running sum passes `u` of the whole, and the sum before it; -1 where nothing weighs anything.  One wavefront; a lane
// takes `per` segments in a row.
struct Found {
  int segment;
  double before, target;
};
template <bool ONE>
__device__ __forceinline__ Found find_segment(const double* sums, int segments, double u) {
  const int lane = threadIdx.x & 63, per = (segments + 63) / 64, first = lane * per, last = min(segments, first + per);
  double own = 0.0;
  const auto sum = [&](int s) { return ONE ? sums[s] : left(sums + s); };
  for (int s = first; s < last; ++s) own += sum(s);
  const double upto = wave_scan(own);
  const double whole = __shfl(upto, 63), prev = __shfl_up(upto, 1);
  Found f = {-1, 0.0, u * whole};
  if (!(whole > 0.0)) return f;
  double run = lane ? prev : 0.0;
  int at = -1, heavy = -1;
  double before = 0.0, heavy_before = 0.0;
  for (int s = first; s < last; ++s) {
    const double x = sum(s), upper = run + x;
    if (x > 0.0) {
      heavy = s;
      heavy_before = run;
      if (at < 0 && upper > f.target) {
        at = s;
        before = run;
      }
    }
    run = upper;
  }
  unsigned long long who = __ballot(at >= 0);
  if (who) {
    const int l = __builtin_ctzll(who);
    f.segment = __shfl(at, l);
    f.before = __shfl(before, l);
  } else {  // (a rounding kept every running sum from passing u W: the last token that weighs anything)
    who = __ballot(heavy >= 0);
    const int l = 63 - __builtin_clzll(who);
    f.segment = __shfl(heavy, l);
    f.before = __shfl(heavy_before, l);
  }
  return f;
}

// The token of segment f.segment at which the running sum passes the target.  One wavefront; a lane takes 16 elements in a row.
template <typename T>
__device__ __forceinline__ long find_token(const Weights<T>& w, const Found& f, int V) {
  constexpr int N = kSegment / 64;
  const int lane = threadIdx.x & 63;
  const long v0 = (long)f.segment * kSegment + lane * N;
  constexpr int E = 16 / sizeof(T);
  double d[N];
  load_weights<T, N / E, E>(w, v0, V, (f.segment + 1l) * kSegment <= V, d);
  double own = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) own += d[j];
  const double upto = wave_scan(own);
  const double prev = __shfl_up(upto, 1);
  double run = f.before + (lane ? prev : 0.0);
  long at = -1, heavy = -1;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    run += d[j];
    if (d[j] > 0.0) {
      heavy = v0 + j;
      if (at < 0 && run > f.target) at = v0 + j;
    }
  }
  unsigned long long who = __ballot(at >= 0);
  if (who) return __shfl(at, __builtin_ctzll(who));
  who = __ballot(heavy >= 0);  // (a rounding at the segment's end: its last token that weighs anything)
  return __shfl(heavy, 63 - __builtin_clzll(who));
}
#endif

}  // namespace tsd
