// tsd_verify_tree_static: a tree of drafted tokens tested against the target's probabilities, or against tokens that the caller chose.
//
// The walk starts at node 0, whose token is the target's already.  At node x the token behind it is drawn from p[x] (draws.h), or is choices[x]; where
// a child of x has it the walk goes on there, else it ends, and the token is the round's last.  A token is kept with probability p[x](token) whatever
// the tree proposes, so that what is committed is distributed as the target's own.
//
// One row of p per step, each behind the one before it: a sequence's workgroup sums the row's segments (16 wavefronts), one of its wavefronts finds the
// segment, the token and the child.  A step takes 2.2 us at 5000 fp32 probabilities, 3.2 at 32000, 4.3 at 50257: of its 9500 clocks there 5800 are the row, 201 KB
// through one compute unit, 2900 the draw (the segment, its second read, two scans), 800 the child and barriers.  In bf16 the row, half the bytes, takes 5800 to 7800
// clocks.  Sums in 32 bits would take 3 % off a call (4 % in bf16): conversions and additions in 64 bits are not what a step waits for.  26 nodes over 32000, walked
// 2 steps: 8.9 us, 64 trees of 32 over 50257, up to 5 steps: 23 us, 16 of them 18, 256, one a compute unit and bound by memory too, 44.
// (Elements looked at one by one 31 us; scans through LDS 30; all wavefronts finding the token for themselves 35.)  Where rows are few and long the
// draws behind all nodes come first (draws_first).
#include <algorithm>

#include "draws.h"
#include "paged_cache.h"

namespace tsd {
namespace {

struct TreeP {
  const void* tokens;  // int32 or int64 [B][N]
  const int* parents;  // [B or 1][N]
  int parents_stride;
  const void* p;       // NULL: choices
  long p_sb, p_sn;
  const float* uniforms;  // [B][N]
  const void* choices;    // [B][N], as tokens, or what was drawn
  const int* n_new;
  int* n_acc;
  void* out;           // [B][N], as tokens
  int* path;           // [B][N]
  int B, N, V, wide, wide_choices;
  int segments;
  int* drawn;          // [B][N]: the draw behind every node, where they come first
};

// A tree in LDS.
struct Nodes {
  long token[kTreeNodes], choice[kTreeNodes];
  int parent[kTreeNodes];
  float uniform[kTreeNodes];
  long drawn[kTreeNodes];  // of the steps so far
  int kept[kTreeNodes];
  int next;
};

// The first child of node x that has this token, or -1.  The same in every lane of a wavefront.
__device__ __forceinline__ int child_of(const Nodes& s, int x, long token, int nodes) {
  const int lane = threadIdx.x & 63;
  for (int base = (x + 1) & ~63; base < nodes; base += 64) {
    const int c = base + lane;
    const unsigned long long who = __ballot(c > x && c < nodes && s.parent[min(c, kTreeNodes - 1)] == x && s.token[min(c, kTreeNodes - 1)] == token);
    if (who) return base + __builtin_ctzll(who);
  }
  return -1;
}

// What 16 bytes of a row's elements have to be for all of them to count as they are: below this, each of them (finite, not negative).
template <typename T>
__device__ __forceinline__ unsigned largest_of(const Words& w) {
  if constexpr (sizeof(T) == 4) {
    return max(max(w[0], w[1]), max(w[2], w[3]));
  } else {
    typedef unsigned short Half2 __attribute__((ext_vector_type(2)));
    Half2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned x = w[i];  // (the cast of a vector's element reads its first)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(Half2, x));
    }
    return (unsigned)max(m[0], m[1]) << 16;
  }
}

// A number from the lanes that CTRL names (0 where there is none, and in rows of 16 lanes that ROWS leaves out).
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
  const uint64_t x = __builtin_bit_cast(uint64_t, v);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive sums over the wavefront's lanes: within rows of 16, then over pairs of rows and halves.
__device__ __forceinline__ double scan(double v) {
  v += moved<0x111, 0xf>(v);  // (row_shr: 1, 2, 4, 8)
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);  // (row_bcast: 15, 31)
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t x = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane));
}

// The weights of a segment that ends behind the row: packs c from element v0 + c * STEP on, 0 beyond V.  Loaded by elements, all on their way together.
template <typename T, int C, int STEP>
__device__ __forceinline__ void load_last(const Weights<T>& w, int v0, int V, double (&d)[C * (16 / sizeof(T))]) {
  constexpr int E = 16 / sizeof(T);
  T x[C * E];
  int first = v0;
  asm volatile("" : "+v"(first));  // (else the addresses are kept in registers, and in memory, for all of the walk)
#pragma unroll
  for (int i = 0; i < C * E; ++i) x[i] = w.p[(unsigned)min(first + i / E * STEP + i % E, V - 1)];
#pragma unroll
  for (int i = 0; i < C * E; ++i) d[i] = v0 + i / E * STEP + i % E < V ? w.of((float)x[i], 0.f, kNoToken) : 0.0;
}

// The sums of a row's segments into LDS, by a whole workgroup: a wavefront takes every so many, the loads of four on their way together.  Weights are
// looked at one by one only where some of a segment's do not count as they are.
template <typename T, int WAVES>
__device__ __forceinline__ void row_sums(const T* p, int V, int segments, double* sums) {
  constexpr int E = 16 / sizeof(T), C = kSegment / (64 * E), U = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Weights<T> w = {p, nullptr, kNoToken};
  const int whole = V / kSegment;
  int i = wave;
  for (; i < whole; i += U * WAVES) {
    Words x[U][C];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * WAVES < whole) {
#pragma unroll
        for (int c = 0; c < C; ++c) x[u][c] = load_pack(p + (unsigned)((i + u * WAVES) * kSegment + (c * 64 + lane) * E));
      }
    __builtin_amdgcn_sched_barrier(0);  // (the loads before all else)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * WAVES >= whole) break;
      unsigned most = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) most = max(most, largest_of<T>(x[u][c]));
      double sum = 0.0;
      if (__any(most >= 0x7F800000u)) {
#pragma unroll
        for (int j = 0; j < C * E; ++j) sum += w.of(element<T>(x[u][j / E], j % E), 0.f, kNoToken);
      } else {
#pragma unroll
        for (int j = 0; j < C * E; ++j) sum += (double)element<T>(x[u][j / E], j % E);
      }
      sum = scan(sum);
      if (lane == 63) sums[i + u * WAVES] = sum;
    }
  }
  if (whole < segments && wave == whole % WAVES) {
    double d[C * E], sum = 0.0;
    load_last<T, C, 64 * E>(w, whole * kSegment + lane * E, V, d);
#pragma unroll
    for (int j = 0; j < C * E; ++j) sum += d[j];
    sum = scan(sum);
    if (lane == 63) sums[whole] = sum;
  }
}

// A draw from a row whose segments' sums are in LDS, as draws.h defines it.  One wavefront, whose scans cross lanes without LDS: a step of the walk waits
// for every one of them.
template <typename T>
__device__ __forceinline__ long draw(const T* p, int V, const double* sums, int segments, float u) {
  const int lane = threadIdx.x & 63, per = (segments + 63) / 64, first = min(segments, lane * per), last = min(segments, first + per);
  // the segment
  double own = 0.0;
  for (int i = first; i < last; ++i) own += sums[i];
  const double upto = scan(own), whole = lane_of(upto, 63), target = (double)u * whole;
  if (!(whole > 0.0)) return -1;
  const double prev = __shfl_up(upto, 1);
  double run = lane ? prev : 0.0, before = 0.0, heavy_before = 0.0;
  int at = -1, heavy = -1;
  for (int i = first; i < last; ++i) {
    const double x = sums[i];
    if (x > 0.0) {
      heavy = i;
      heavy_before = run;
      if (at < 0 && run + x > target) {
        at = i;
        before = run;
      }
    }
    run += x;
  }
  unsigned long long who = __ballot(at >= 0);
  const bool passed = who != 0;  // (else a rounding kept every running sum from passing u W: the last token that weighs anything)
  if (!passed) who = __ballot(heavy >= 0);
  const int l = passed ? __builtin_ctzll(who) : 63 - __builtin_clzll(who);
  const int segment = __builtin_amdgcn_readlane(passed ? at : heavy, l);
  const double base = lane_of(passed ? before : heavy_before, l);
  // the token in it: a lane takes N elements in a row
  constexpr int N = kSegment / 64, E = 16 / sizeof(T);
  const Weights<T> w = {p, nullptr, kNoToken};
  const int v0 = segment * kSegment + lane * N;
  double d[N];
  if ((segment + 1) * kSegment <= V) {  // (the same in every lane)
    Words x[N / E];
    unsigned most = 0;
#pragma unroll
    for (int c = 0; c < N / E; ++c) x[c] = load_pack(p + (unsigned)(v0 + c * E));
#pragma unroll
    for (int c = 0; c < N / E; ++c) most = max(most, largest_of<T>(x[c]));
    const bool odd = __any(most >= 0x7F800000u);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float y = element<T>(x[j / E], j % E);
      d[j] = odd ? w.of(y, 0.f, kNoToken) : (double)y;
    }
  } else {
    load_last<T, N / E, E>(w, v0, V, d);
  }
  own = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) own += d[j];
  const double sum = __shfl_up(scan(own), 1);
  run = base + (lane ? sum : 0.0);
  unsigned over = 0, some = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    run += d[j];
    some |= d[j] > 0.0 ? 1u << j : 0u;
    over |= run > target ? 1u << j : 0u;
  }
  over &= some;
  who = __ballot(over);
  if (who) {
    const int l = __builtin_ctzll(who);
    return segment * kSegment + l * N + __builtin_ctz(__builtin_amdgcn_readlane(over, l));
  }
  who = __ballot(some);  // (a rounding at the segment's end: its last token that weighs anything)
  const int k = 63 - __builtin_clzll(who);
  return segment * kSegment + k * N + 31 - __builtin_clz(__builtin_amdgcn_readlane(some, k));
}

template <typename T>
__device__ __forceinline__ const T* row_of(const TreeP& a, int b, int node) {
  return reinterpret_cast<const T*>(a.p) + b * a.p_sb + node * a.p_sn;
}

// The draws behind all nodes, a workgroup each: a node's step is its depth below the root.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void draw_nodes_kernel(const TreeP a) {
  extern __shared__ double sums[];  // [segments]
  __shared__ int parent[kTreeNodes];
  const int b = blockIdx.x / a.N, node = blockIdx.x - b * a.N;
  if (node >= (a.n_new ? a.n_new[b] : a.N)) return;
  for (int i = threadIdx.x; i <= node; i += WAVES * 64) parent[i] = a.parents[(long)b * a.parents_stride + i];
  __syncthreads();
  int depth = 0;
  for (int x = node; x > 0; ++depth) {
    const int up = parent[x];
    if (up < 0 || up >= x) return;  // (does not hang on the root)
    x = up;
  }
  const T* p = row_of<T>(a, b, node);
  const float u = a.uniforms[(long)b * a.N + depth];
  row_sums<T, WAVES>(p, a.V, a.segments, sums);
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const long token = draw(p, a.V, sums, a.segments, u);
  if (threadIdx.x == 0) a.drawn[(long)b * a.N + node] = (int)token;
}

// T: void for chosen tokens.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void verify_tree_kernel(const TreeP a) {
  extern __shared__ double sums[];  // [segments]
  __shared__ Nodes s;
  const int b = blockIdx.x;
  const int nodes = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  for (int i = threadIdx.x; i < nodes; i += WAVES * 64) {
    s.token[i] = token_at(a.tokens, (long)b * a.N + i, a.wide);
    s.parent[i] = a.parents[(long)b * a.parents_stride + i];
    if constexpr (std::is_void_v<T>)
      s.choice[i] = token_at(a.choices, (long)b * a.N + i, a.wide_choices);
    else
      s.uniform[i] = a.uniforms[(long)b * a.N + i];
  }
  __syncthreads();
  int n = 0;
  for (int at = 0; at >= 0 && n < nodes; ++n) {
    if constexpr (!std::is_void_v<T>) {
      row_sums<T, WAVES>(row_of<T>(a, b, at), a.V, a.segments, sums);
      __syncthreads();
    }
    if (threadIdx.x < 64) {  // (one wavefront: sixteen that do the same take turns)
      long token;
      if constexpr (std::is_void_v<T>)
        token = s.choice[at];
      else
        token = draw(row_of<T>(a, b, at), a.V, sums, a.segments, s.uniform[n]);
      const int next = token < 0 ? -1 : child_of(s, at, token, nodes);
      if (threadIdx.x == 0) {
        s.drawn[n] = token;
        s.kept[n] = at;
        s.next = next;
      }
      if constexpr (WAVES == 1) at = next;
    }
    if constexpr (WAVES > 1) {
      __syncthreads();
      at = __builtin_amdgcn_readfirstlane(s.next);  // (the row's address is scalar)
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.N; i += WAVES * 64) {
    const long o = (long)b * a.N + i, x = i < n ? s.drawn[i] : -1;
    if (a.wide)
      reinterpret_cast<long*>(a.out)[o] = x;
    else
      reinterpret_cast<int*>(a.out)[o] = (int)x;
    a.path[o] = i < n ? s.kept[i] : -1;
  }
  if (threadIdx.x == 0) a.n_acc[b] = n - 1;
}

constexpr int kMostWords = 1 << 21;  // of a vocabulary: the sums of a row's segments, 16 KB, in LDS

int check_tree(int dtype, int32_t B, int32_t N, int32_t V) {
  if (dtype != TSD_F32 && dtype != TSD_BF16) return fail_no_handle(TSD_E_INVALID_ARG, "dtype must be TSD_F32 or TSD_BF16");
  if (B < 1 || N < 1 || V < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1, N >= 1, V >= 1");
  if (N > kTreeNodes) return fail_no_handle(TSD_E_OUT_OF_RANGE, "a tree has at most 256 nodes");
  if (V > kMostWords) return fail_no_handle(TSD_E_OUT_OF_RANGE, "V beyond 2^21");
  if (B > max_workgroups(1024)) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B beyond what a launch takes");
  return TSD_OK;
}

// Whether the draws behind all nodes come first, side by side, and then the walk: where rows are so long that a step takes more than a second launch, and all of
// them are no more to read than the time saved.  us so and step by step (fp32, trees walked 2 steps on average, 5 at most): 26 nodes, 131072 x 1 13.6, 19.8,
// x 8 27.5, 28.0; 32000 x 1 11.0, 9.0, x 8 12.2, 13.9, x 16 19.5, 15.4; 32 nodes, 50257 x 64 66.8, 24.1.
bool draws_first(int32_t B, int32_t N, int32_t V, int32_t dtype) {
  return V > 65536 && (int64_t)B * N * V * type_bytes(dtype) <= 64 << 20;
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_verify_tree_workspace(int32_t B, int32_t N, int32_t V, int32_t dtype, size_t* bytes_host) {
  const int rc = check_tree(dtype, B, N, V);
  if (rc) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  *bytes_host = draws_first(B, N, V, dtype) ? (size_t)B * N * 4 : 0;
  return TSD_OK;
}

extern "C" int tsd_verify_tree_static(const void* tokens_dev, const int32_t* parents_dev, int32_t parents_stride, const void* p_dev, int32_t dtype,
                                      int32_t token_bytes, int32_t B, int32_t N, int32_t V, int64_t p_stride_b, int64_t p_stride_n,
                                      const float* uniforms_dev, const void* choices_dev, const int32_t* n_new_dev, int32_t* n_acc_dev, void* out_dev,
                                      int32_t* path_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int rc = tsd_verify_tree_workspace(B, N, p_dev ? V : 1, p_dev ? dtype : TSD_F32, &need);
  if (rc) return rc;
  if (!p_dev) need = 0;
  if (!tokens_dev || !parents_dev || !n_acc_dev || !out_dev || !path_dev)
    return fail_no_handle(TSD_E_INVALID_ARG, "tokens_dev, parents_dev, n_acc_dev, out_dev and path_dev must not be NULL");
  if (!p_dev == !choices_dev) return fail_no_handle(TSD_E_INVALID_ARG, "needs either p_dev or choices_dev");
  if (p_dev && !uniforms_dev) return fail_no_handle(TSD_E_INVALID_ARG, "uniforms_dev must not be NULL beside p_dev");
  if (token_bytes != 4 && token_bytes != 8) return fail_no_handle(TSD_E_INVALID_ARG, "token_bytes must be 4 or 8");
  if (parents_stride && parents_stride < N) return fail_no_handle(TSD_E_INVALID_ARG, "parents_stride must be 0 or at least N");
  if (p_dev && (p_stride_b < 0 || p_stride_n < 0)) return fail_no_handle(TSD_E_INVALID_ARG, "strides must not be negative");
  if (need && (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 3)))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that tsd_verify_tree_workspace gives for these sizes, 4-byte aligned");
  TreeP a;
  a.tokens = tokens_dev;
  a.parents = parents_dev;
  a.parents_stride = parents_stride;
  a.p = p_dev;
  a.p_sb = p_stride_b;
  a.p_sn = p_stride_n;
  a.uniforms = uniforms_dev;
  a.choices = choices_dev;
  a.n_new = n_new_dev;
  a.n_acc = n_acc_dev;
  a.out = out_dev;
  a.path = path_dev;
  a.B = B;
  a.N = N;
  a.V = V;
  a.wide = a.wide_choices = token_bytes == 8;
  a.segments = p_dev ? (int)((V + (int64_t)kSegment - 1) / kSegment) : 0;
  a.drawn = static_cast<int*>(workspace_dev);
  const hipStream_t st = (hipStream_t)stream;
  const size_t lds = (size_t)a.segments * 8;
  const auto walk = [&](auto type) {
    using T = decltype(type);
    if (need)
      draw_nodes_kernel<T, 16><<<(unsigned)((int64_t)B * N), 1024, lds, st>>>(a);
    else
      verify_tree_kernel<T, 16><<<B, 1024, lds, st>>>(a);
  };
  if (p_dev) dtype == TSD_BF16 ? walk(bf16()) : walk(float());
  if (p_dev && need) {
    a.choices = a.drawn;
    a.wide_choices = false;
  }
  if (!p_dev || need) verify_tree_kernel<void, 1><<<B, 64, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("tree verification launch: ") + hipGetErrorString(e));
}
