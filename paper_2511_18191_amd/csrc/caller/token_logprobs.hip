// tsd_token_logprobs_static: log probability of a given token, entropy, and the likeliest tokens, from logits.
//
// With d_v = (x_v - m) / temperature, m a maximum so far: S = sum e^d, W = sum d e^d; a larger m' takes them to f S and f (W + S (m - m') / temperature),
// f = e^((m - m') / temperature).  Then log p_v = d_v - ln S and the entropy is ln S - W / S, two numbers that are not negative: nothing cancels.  (Differences to
// the maximum itself are taken before the factor: logits may be as large as their type's largest.  They are taken of quarters, and the factor is four times
// as large: so are the temperatures, and neither the difference nor the factor leaves the normal numbers.  Quarters round as the whole do: same bits.)
//
// One pass over the row.  For the alternatives each lane's maxima of kCell elements stay in LDS.  A bound that at least `top` elements reach is had
// by counting: of the maxima of all lanes, in fours, it is the top-th.  Only cells that reach it are read again (some
// top of them, out of the last cache), and what reaches it there, a few more than top, is ranked by counting too.  Where more elements reach the bound than
// LDS has room for (masks of one finite value, say), those above it and then as many at it as are needed, in the order of the row; where that does
// not fit either, one after the other.
//
// A row takes one workgroup, or, where long rows are few, several; the one that comes last joins their sums and lists (last_arriver.h).
//
// Many rows are memory bound: 1024 rows of 131072 bf16 logits 52.6 us without alternatives, 5.1 TB/s (what a copy reaches), 59 us with twenty, whose bounds
// and second looks are not hidden in full.  A row of 32000 fp32: 6.6 us, and 9.3 with five alternatives; the launch, two trips to memory, and for
// alternatives a third behind four barriers.  (1024 lanes a workgroup: 7.9 and 14; bounds from every wavefront's sorted maxima: 10.3.)
#include <algorithm>
#include <cmath>

#include "draws.h"
#include "paged_cache.h"

namespace tsd {
namespace {

constexpr int kLanes = 256;                  // of a workgroup
constexpr int kCell = 64;                    // elements of a lane whose maximum is kept
constexpr int kMostPart = 262144;            // elements of a workgroup: its maxima are in LDS
constexpr int kMostTop = 32;
constexpr int kMostGroups = 32;              // workgroups of a row
constexpr int kMostCells = 512, kMostFound = 1024;  // cells and elements that reach the bound, in LDS

struct ScoreP {
  const void* logits;
  long sb, st;
  const void* tokens;  // int32 or int64 [B][T], or NULL
  const int* n_new;
  int B, T, V, top, wide;
  float inv4, scale4;  // 4 / temperature, and times log2 e (of quarters: base e, base 2)
  float *logprobs, *entropy, *top_logprobs;
  int* top_ids;
  int groups, per;     // workgroups of a row, and the elements that each of them takes
  float* sums;         // [rows][groups][4]: m, S, W (in base 2) (groups > 1)
  uint64_t* lists;     // [rows][groups][top]
  uint64_t* slots;     // [rows][groups]
  uint64_t tag;
};

// Sums of a part of a row, relative to its maximum; W in base 2.
struct Sums {
  float m, s, w;
};
constexpr Sums kNoSums = {-INFINITY, 0.f, 0.f};

// A quarter of a difference.
__device__ __forceinline__ float quarter(float a, float b) { return fmaf(a, 0.25f, -0.25f * b); }

// What sums relative to `from` change by, relative to `to` >= from: the factor's exponent.
__device__ __forceinline__ float shift_of(float from, float to, float scale4) { return from == -INFINITY ? 0.f : quarter(from, to) * scale4; }

__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float scale4) {
  Sums r;
  r.m = fmaxf(a.m, b.m);
  const float da = shift_of(a.m, r.m, scale4), db = shift_of(b.m, r.m, scale4);
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  r.s = fa * a.s + fb * b.s;
  r.w = fa * fmaf(a.s, fmaxf(da, -200.f), a.w) + fb * fmaf(b.s, fmaxf(db, -200.f), b.w);
  return r;
}

// An element and its index as one number: the larger value first, then the lower index.
__device__ __forceinline__ uint64_t key_of(float x, unsigned i) {
  const unsigned u = __float_as_uint(x + 0.f);  // (-0 and 0 are the same)
  return (uint64_t)(u ^ (unsigned)((int)u >> 31 | (int)0x80000000)) << 32 | ~i;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const unsigned s = (unsigned)(key >> 32);
  return __uint_as_float(s & 0x80000000u ? s ^ 0x80000000u : ~s);
}
__device__ __forceinline__ unsigned index_of(uint64_t key) { return ~(unsigned)key; }

// N elements x[] of a lane into its sums.  Returns the largest.
template <int N>
__device__ __forceinline__ float take(Sums& a, const float (&x)[N], float scale4) {
  float mx = x[0];
#pragma unroll
  for (int j = 1; j < N; ++j) mx = fmaxf(mx, x[j]);
  const float m = fmaxf(a.m, mx), from = m == -INFINITY ? 0.f : m;
  const float d = shift_of(a.m, m, scale4), f = __builtin_amdgcn_exp2f(d);
  a.w = f * fmaf(a.s, fmaxf(d, -200.f), a.w);
  a.s *= f;
  a.m = m;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float t = quarter(x[j], from) * scale4, e = __builtin_amdgcn_exp2f(t);  // (a NaN, or an infinite maximum, makes S a NaN)
    a.s += e;
    a.w = fmaf(e, fmaxf(t, -200.f), a.w);  // (e is 0 there, and t may be infinite)
  }
  return mx;
}

// A part of a row as a workgroup goes over it: element ((i * C + c) * kLanes + lane) * E + e of it is element e of load c of cell (i, lane).
template <typename T>
struct Part {
  static constexpr int E = 16 / sizeof(T), C = kCell / E;
  const T* p;
  int n;
  __device__ __forceinline__ int start(int i, int c, int lane) const { return ((i * C + c) * kLanes + lane) * E; }
  // Element l of a cell.
  __device__ __forceinline__ int place(int cell, int l) const { return start(cell / kLanes, l / E, cell % kLanes) + l % E; }
};

// Loads c0 .. c0 + U - 1 of cell i of the lane.
template <typename T, int U>
__device__ __forceinline__ void load_cells(const Part<T>& q, int i, int c0, float (&x)[U * Part<T>::E]) {
  constexpr int E = Part<T>::E;
  if (q.start(i, c0 + U, 0) <= q.n) {  // (all of them are there, in every lane)
    Words y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) y[u] = load_pack(q.p + q.start(i, c0 + u, threadIdx.x));
#pragma unroll
    for (int j = 0; j < U * E; ++j) x[j] = element<T>(y[j / E], j % E);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = q.start(i, c0 + u, threadIdx.x);
      if (q.start(i, c0 + u + 1, 0) <= q.n) {
        const Words y = load_pack(q.p + at);
#pragma unroll
        for (int e = 0; e < E; ++e) x[u * E + e] = element<T>(y, e);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x[u * E + e] = -INFINITY;
          if (at + e < q.n) x[u * E + e] = (float)q.p[at + e];
        }
      }
    }
  }
}

// The `top` largest of n keys in LDS, ranked: put(rank, key).
template <typename Put>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int top, Put put) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const uint64_t own = keys[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += keys[j] > own;
    if (rank < top) put(rank, own);
  }
}

// What finding the alternatives needs in LDS.
struct Candidates {
  uint64_t keys[kMostFound];
  int cells[kMostCells];
  int n_cells, n_found, ties[kLanes / 64];
  uint64_t best[kLanes / 64];
  float maxima[kLanes / 4];
  float bound;
};

// The elements of cells that reach `bound` (above: exceed it) into LDS, whose counts are 0; whether they fit.
template <typename T>
__device__ __forceinline__ bool collect(const Part<T>& q, long base, const float* maxima, int blocks, float bound, bool above, Candidates& f) {
  const auto in = [&](float x) { return above ? x > bound : x >= bound && x > -INFINITY; };
  for (int i = threadIdx.x; i < blocks * kLanes; i += kLanes)
    if (in(maxima[i])) {
      const int at = atomicAdd(&f.n_cells, 1);
      if (at < kMostCells) f.cells[at] = i;
    }
  __syncthreads();
  if (f.n_cells > kMostCells) return false;
  constexpr int U = 8;  // loads on their way together
  const int n = f.n_cells * kCell;
  for (int i0 = threadIdx.x; i0 < n; i0 += U * kLanes) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * kLanes, n - 1), at = q.place(f.cells[i / kCell], i % kCell);
      x[u] = (float)q.p[min(at, q.n - 1)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kLanes;
      if (i >= n || !in(x[u])) continue;
      const int at = q.place(f.cells[i / kCell], i % kCell);
      if (at >= q.n) continue;
      const int to = atomicAdd(&f.n_found, 1);
      if (to < kMostFound) f.keys[to] = key_of(x[u], (unsigned)(base + at));
    }
  }
  __syncthreads();
  return f.n_found <= kMostFound;
}

// Adds the first `want` elements equal to `bound`, in the order of the row, to the keys in LDS (as many as `top` in all).
template <typename T>
__device__ __forceinline__ void collect_ties(const Part<T>& q, long base, float bound, int want, Candidates& f) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int at0 = 0; at0 < q.n && want > 0; at0 += kLanes) {
    const int at = at0 + threadIdx.x;
    const bool tie = at < q.n && (float)q.p[at] == bound;
    const unsigned long long who = __ballot(tie);
    __syncthreads();
    if (lane == 0) f.ties[wave] = __popcll(who);
    __syncthreads();
    int before = __popcll(who & ((1ull << lane) - 1)), all = 0;
    for (int v = 0; v < kLanes / 64; ++v) {
      if (v < wave) before += f.ties[v];
      all += f.ties[v];
    }
    if (tie && before < want) f.keys[f.n_found + before] = key_of(bound, (unsigned)(base + at));
    const int more = min(all, want);
    __syncthreads();
    if (threadIdx.x == 0) f.n_found += more;
    want -= more;
  }
  __syncthreads();
}

// The `top` largest elements one after the other.
template <typename T>
__device__ __forceinline__ void extract(const Part<T>& q, long base, int top, Candidates& f) {
  uint64_t last = ~0ull;
  int n = 0;
  for (; n < top; ++n) {
    uint64_t best = 0;
    for (int at = threadIdx.x; at < q.n; at += kLanes) {
      const float x = (float)q.p[at];
      const uint64_t key = x > -INFINITY ? key_of(x, (unsigned)(base + at)) : 0;
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) f.best[threadIdx.x >> 6] = best;
    __syncthreads();
    for (int v = 0; v < kLanes / 64; ++v) best = max(best, f.best[v]);
    if (!best) break;
    if (threadIdx.x == 0) f.keys[n] = best;
    last = best;
  }
  __syncthreads();
  if (threadIdx.x == 0) f.n_found = n;
  __syncthreads();
}

// The part's elements among which its `top` largest are, as keys in LDS.
template <typename T>
__device__ __forceinline__ void find_top(const Part<T>& q, long base, const float* maxima, int blocks, float lane_max, int top, Candidates& f) {
  static_assert(kLanes / 4 == 64);
  lane_max = fmaxf(lane_max, __shfl_xor(lane_max, 1));
  lane_max = fmaxf(lane_max, __shfl_xor(lane_max, 2));
  if ((threadIdx.x & 3) == 0) f.maxima[threadIdx.x >> 2] = lane_max;
  __syncthreads();
  if (threadIdx.x < 64) {  // (the largest value that at least `top` of the 64 reach)
    const float own = f.maxima[threadIdx.x];
    int reach = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) reach += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own), j)) >= own;
    float b = reach >= top ? own : -INFINITY;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) b = fmaxf(b, __shfl_xor(b, o));
    if (threadIdx.x == 0) {
      f.bound = b;
      f.n_cells = f.n_found = 0;
    }
  }
  __syncthreads();
  const float bound = f.bound;
  if (collect(q, base, maxima, blocks, bound, false, f)) return;
  if (bound > -INFINITY) {
    __syncthreads();
    if (threadIdx.x == 0) f.n_cells = f.n_found = 0;
    __syncthreads();
    if (collect(q, base, maxima, blocks, bound, true, f)) {
      collect_ties(q, base, bound, top - f.n_found, f);
      return;
    }
  }
  extract(q, base, top, f);
}

// A row's results.  One lane.
__device__ __forceinline__ void put_row(const ScoreP& a, long row, const Sums& z, float x, bool there) {
  const bool none = z.s == 0.f;  // no token weighs anything
  const float ln_s = logf(z.s);
  if (a.logprobs) a.logprobs[row] = none || !there ? (z.s != z.s ? z.s : -INFINITY) : quarter(x, z.m) * a.inv4 - ln_s;
  a.entropy[row] = none ? 0.f : ln_s - z.w / z.s * 0.69314718055994531f;
}
// The likeliest of the keys in LDS.
__device__ __forceinline__ void put_top(const ScoreP& a, long row, const Sums& z, const Candidates& f) {
  rank_keys(f.keys, f.n_found, a.top, [&](int rank, uint64_t key) {
    a.top_ids[row * a.top + rank] = (int)index_of(key);
    a.top_logprobs[row * a.top + rank] = quarter(value_of(key), z.m) * a.inv4 - logf(z.s);
  });
  if (threadIdx.x >= f.n_found && threadIdx.x < a.top) {
    a.top_ids[row * a.top + threadIdx.x] = -1;
    a.top_logprobs[row * a.top + threadIdx.x] = -INFINITY;
  }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kLanes) void token_logprobs_kernel(const ScoreP a) {
  extern __shared__ float maxima[];  // [blocks][kLanes] (TOP)
  __shared__ Sums parts[kLanes / 64];
  __shared__ std::conditional_t<TOP, Candidates, int> found;
  const int row_at = blockIdx.x / a.groups, group = blockIdx.x - row_at * a.groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = row_at / a.T, t = row_at - b * a.T;
  const long row = row_at;
  if (a.n_new && t >= a.n_new[b]) {  // (not read)
    if (group) return;
    if (threadIdx.x == 0) {
      if (a.logprobs) a.logprobs[row] = 0.f;
      a.entropy[row] = 0.f;
    }
    if (TOP && threadIdx.x < a.top) {
      a.top_ids[row * a.top + threadIdx.x] = -1;
      a.top_logprobs[row * a.top + threadIdx.x] = 0.f;
    }
    return;
  }
  const T* whole = reinterpret_cast<const T*>(a.logits) + b * a.sb + t * a.st;
  const long token = a.tokens ? token_at(a.tokens, row, a.wide) : -1;
  const bool there = token >= 0 && token < a.V;
  const float x_token = there ? (float)whole[token] : 0.f;

  const long base = (long)group * a.per;
  const Part<T> q = {whole + base, (int)min((long)a.per, a.V - base)};
  const int blocks = (q.n + kLanes * kCell - 1) / (kLanes * kCell);
  constexpr int U = 8, N = U * Part<T>::E;
  Sums z = kNoSums;
  for (int i = 0; i < blocks; ++i) {
    float cell = -INFINITY;
#pragma unroll
    for (int c0 = 0; c0 < Part<T>::C; c0 += U) {
      if (q.start(i, c0, 0) >= q.n) break;
      float x[N];
      load_cells<T, U>(q, i, c0, x);
      cell = fmaxf(cell, take(z, x, a.scale4));
    }
    if (TOP) maxima[i * kLanes + threadIdx.x] = cell;
  }
  const float lane_max = z.m;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    Sums y;
    y.m = __shfl_xor(z.m, o);
    y.s = __shfl_xor(z.s, o);
    y.w = __shfl_xor(z.w, o);
    z = join(z, y, a.scale4);
  }
  if (lane == 0) parts[wave] = z;
  __syncthreads();
  z = parts[0];
#pragma unroll
  for (int v = 1; v < kLanes / 64; ++v) z = join(z, parts[v], a.scale4);
  if constexpr (TOP) find_top(q, base, maxima, blocks, lane_max, a.top, found);

  if (a.groups == 1) {
    if (threadIdx.x == 0) put_row(a, row, z, x_token, there);
    if constexpr (TOP) put_top(a, row, z, found);
    return;
  }
  const long at = row * a.groups + group;
  if (threadIdx.x == 0) {
    leave(a.sums + at * 4, z.m);
    leave(a.sums + at * 4 + 1, z.s);
    leave(a.sums + at * 4 + 2, z.w);
  }
  if constexpr (TOP) {
    rank_keys(found.keys, found.n_found, a.top, [&](int rank, uint64_t key) { leave(a.lists + at * a.top + rank, key); });
    if (threadIdx.x >= found.n_found && threadIdx.x < a.top) leave(a.lists + at * a.top + threadIdx.x, (uint64_t)0);
  }
  uint64_t* slots = a.slots + row * a.groups;
  if (!came_last(slots, a.groups, group, a.tag)) return;
  z = kNoSums;
  if (lane < a.groups) {
    const float* from = a.sums + (row * a.groups + lane) * 4;
    z.m = left(from);
    z.s = left(from + 1);
    z.w = left(from + 2);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    Sums y;
    y.m = __shfl_xor(z.m, o);
    y.s = __shfl_xor(z.s, o);
    y.w = __shfl_xor(z.w, o);
    z = join(z, y, a.scale4);
  }
  if (threadIdx.x == 0) put_row(a, row, z, x_token, there);
  if constexpr (TOP) {
    // The lists' heads, 64 in all, give a bound that at least `top` keys reach; those are ranked.
    Candidates& f = found;
    const uint64_t* lists = a.lists + row * a.groups * a.top;
    const int n = a.groups * a.top;
    constexpr int U = kMostFound / kLanes;
    uint64_t key[U];
#pragma unroll
    for (int u = 0; u < U; ++u) key[u] = u * kLanes < n ? left(lists + min(u * kLanes + (int)threadIdx.x, n - 1)) : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * kLanes + threadIdx.x >= n) key[u] = 0;
      if (u * kLanes < n) f.keys[u * kLanes + threadIdx.x] = key[u];
    }
    if (threadIdx.x == 0) f.n_found = 0;
    __syncthreads();
    if (wave == 0) {
      const int heads = min(a.top, 64 / a.groups), g = lane / heads;
      const uint64_t own = g < a.groups ? f.keys[g * a.top + lane - g * heads] : 0;
      int reach = 0;
#pragma unroll
      for (int j = 0; j < 64; ++j)
        reach += ((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(own >> 32), j) << 32 | (unsigned)__builtin_amdgcn_readlane((int)own, j)) >= own;
      uint64_t b = reach < a.top ? 0 : own;
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) b = max(b, (uint64_t)__shfl_xor((unsigned long long)b, o));
      if (lane == 0) f.best[0] = b;
    }
    __syncthreads();
    const uint64_t bound = f.best[0];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (key[u] && key[u] >= bound) f.keys[atomicAdd(&f.n_found, 1)] = key[u];
    __syncthreads();
    put_top(a, row, z, f);
  }
  clear_slots(slots, a.groups);
}

// Workgroups of a row: one, but for long rows that are few, whose join (4 us) pays: then some 512 in all, with 8192 elements at least.  us with 1, 4, 8 and 16 a
// row (fp32, five alternatives): 32000 x 1 row 9.3, 10.4, 11.6, 11.7, x 256 12.1, 18.0, 26.6, 42.0; 131072 x 1 17.1, 12.6, 12.0, 11.3, x 64 20.9,
// 16.0, 16.1, 17.7, x 128 26.5, 22.3, 23.1, 27.6, x 256 29.5, 35.0, 38.9, 43.4; 262144 x 1 34.1, 15.3, 13.4, 12.0.
struct ScorePlan {
  int groups, per;
};
ScorePlan score_plan(int64_t rows, int V) {
  int64_t want = V <= 65536 || rows >= 192 ? 1 : std::min<int64_t>({16, V / 8192, 512 / rows});
  want = std::max(want, (V + (int64_t)kMostPart - 1) / kMostPart);
  ScorePlan s;
  s.per = (int)((V + want - 1) / want + 1023) / 1024 * 1024;
  s.groups = (V + s.per - 1) / s.per;
  return s;
}
constexpr int kMostTokensScored = kMostPart * kMostGroups;

int check_scores(int32_t B, int32_t T, int32_t V, int32_t top) {
  if (B < 1 || T < 1 || V < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1, T >= 1 and V >= 1");
  if (top < 0) return fail_no_handle(TSD_E_INVALID_ARG, "top must not be negative");
  if (top > kMostTop) return fail_no_handle(TSD_E_OUT_OF_RANGE, "at most 32 alternatives");
  if (V > kMostTokensScored) return fail_no_handle(TSD_E_OUT_OF_RANGE, "V beyond 2^23");
  const int64_t rows = (int64_t)B * T;
  if (rows > max_workgroups(kLanes) || rows * score_plan(rows, V).groups > max_workgroups(kLanes)) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B * T beyond what a launch takes");
  return TSD_OK;
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_token_logprobs_workspace(int32_t B, int32_t T, int32_t V, int32_t top, size_t* bytes_host) {
  const int rc = check_scores(B, T, V, top);
  if (rc) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  const int64_t rows = (int64_t)B * T;
  const ScorePlan s = score_plan(rows, V);
  *bytes_host = s.groups == 1 ? 0 : (size_t)rows * s.groups * (16 + 8 * (size_t)top + 8);
  return TSD_OK;
}

extern "C" int tsd_token_logprobs_static(const void* logits_dev, int32_t dtype, int32_t token_bytes, int32_t B, int32_t T, int32_t V, int64_t stride_b,
                                         int64_t stride_t, const void* tokens_dev, const int32_t* n_new_dev, float temperature, int32_t top,
                                         float* logprobs_dev, float* entropy_dev, int32_t* top_ids_dev, float* top_logprobs_dev,
                                         void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int rc = tsd_token_logprobs_workspace(B, T, V, top, &need);
  if (rc) return rc;
  if (dtype != TSD_F32 && dtype != TSD_BF16) return fail_no_handle(TSD_E_INVALID_ARG, "dtype must be TSD_F32 or TSD_BF16");
  if (!logits_dev || !entropy_dev) return fail_no_handle(TSD_E_INVALID_ARG, "logits_dev and entropy_dev must not be NULL");
  if (!tokens_dev != !logprobs_dev) return fail_no_handle(TSD_E_INVALID_ARG, "tokens_dev and logprobs_dev go together");
  if (tokens_dev && token_bytes != 4 && token_bytes != 8) return fail_no_handle(TSD_E_INVALID_ARG, "token_bytes must be 4 or 8");
  if (top && (!top_ids_dev || !top_logprobs_dev)) return fail_no_handle(TSD_E_INVALID_ARG, "top_ids_dev and top_logprobs_dev must not be NULL beside top");
  if (stride_b < 0 || stride_t < 0) return fail_no_handle(TSD_E_INVALID_ARG, "strides must not be negative");
  if (!(temperature >= 1e-6f) || !std::isfinite(temperature)) return fail_no_handle(TSD_E_INVALID_ARG, "temperature must be finite, at least 1e-6");
  if (need && (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 7)))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that tsd_token_logprobs_workspace gives for these sizes, 8-byte aligned");
  const int64_t rows = (int64_t)B * T;
  const ScorePlan s = score_plan(rows, V);
  ScoreP a;
  a.logits = logits_dev;
  a.sb = stride_b;
  a.st = stride_t;
  a.tokens = tokens_dev;
  a.n_new = n_new_dev;
  a.B = B;
  a.T = T;
  a.V = V;
  a.top = top;
  a.wide = token_bytes == 8;
  a.inv4 = (float)(4.0 / temperature);
  a.scale4 = (float)(4.0 * 1.4426950408889634 / temperature);
  a.logprobs = logprobs_dev;
  a.entropy = entropy_dev;
  a.top_ids = top_ids_dev;
  a.top_logprobs = top_logprobs_dev;
  a.groups = s.groups;
  a.per = s.per;
  a.lists = static_cast<uint64_t*>(workspace_dev);
  a.slots = a.lists + (size_t)rows * s.groups * top;
  a.sums = reinterpret_cast<float*>(a.slots + (size_t)rows * s.groups);
  a.tag = s.groups > 1 ? new_tag() : 0;
  const hipStream_t st = (hipStream_t)stream;
  const unsigned grid = (unsigned)(rows * s.groups);
  const size_t lds = top ? (size_t)((s.per + kLanes * kCell - 1) / (kLanes * kCell)) * kLanes * 4 : 0;
  const auto go = [&](auto with, auto without) { (top ? with : without)<<<grid, kLanes, lds, st>>>(a); };
  if (dtype == TSD_BF16)
    go(token_logprobs_kernel<bf16, true>, token_logprobs_kernel<bf16, false>);
  else
    go(token_logprobs_kernel<float, true>, token_logprobs_kernel<float, false>);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("token scores launch: ") + hipGetErrorString(e));
}
