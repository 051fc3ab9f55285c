// tsd_verify_tree_static: a tree of drafted tokens tested against the target's probabilities, or against tokens that the caller chose.
//
// The walk starts at node 0, whose token is the target's already.  At node x the token behind it is drawn from p[x] (draws.h), or is choices[x]; where
// a child of x has it the walk goes on there, else it ends, and the token is the round's last.  A token is kept with probability p[x](token) whatever
// the tree proposes, so that what is committed is distributed as the target's own.
//
// One row of p per step, each behind the one before it: a sequence's workgroup sums the row's segments (16 wavefronts), finds the token, then the child.
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
  const void* choices;    // [B][N], as tokens
  const int* n_new;
  int* n_acc;
  void* out;           // [B][N], as tokens
  int* path;           // [B][N]
  int B, N, V, wide;
  int segments;
};

// A tree in LDS.
struct Nodes {
  long token[kTreeNodes];
  int parent[kTreeNodes];
  long drawn[kTreeNodes];  // of the steps so far
  int kept[kTreeNodes];
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

// T: void for chosen tokens.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void verify_tree_kernel(const TreeP a) {
  extern __shared__ double sums[];  // [2][segments]: of two steps in turn
  __shared__ Nodes s;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nodes = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  for (int i = threadIdx.x; i < nodes; i += WAVES * 64) {
    s.token[i] = token_at(a.tokens, (long)b * a.N + i, a.wide);
    s.parent[i] = a.parents[(long)b * a.parents_stride + i];
  }
  __syncthreads();
  int n = 0;
  for (int at = 0; n < nodes; ++n) {
    long token;
    if constexpr (std::is_void_v<T>) {
      token = token_at(a.choices, (long)b * a.N + at, a.wide);
    } else {
      const Weights<T> w = {reinterpret_cast<const T*>(a.p) + b * a.p_sb + at * a.p_sn, nullptr, kNoToken};
      double* own = sums + (n & 1) * a.segments;
      for (int i = wave; i < a.segments; i += WAVES) {
        const double sum = segment_sum(w, i, a.V);
        if (lane == 0) own[i] = sum;
      }
      __syncthreads();  // (the wavefronts that still look at the former step's sums do not have to be waited for: there are two)
      const Found f = find_segment<true>(own, a.segments, (double)a.uniforms[(long)b * a.N + n]);
      token = f.segment < 0 ? -1 : find_token(w, f, a.V);
    }
    if (threadIdx.x == 0) {
      s.drawn[n] = token;
      s.kept[n] = at;
    }
    at = token < 0 ? -1 : child_of(s, at, token, nodes);
    if (at < 0) {
      ++n;
      break;
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

constexpr int kMostWords = 1 << 21;  // of a vocabulary: the sums of a row's segments, twice, in LDS

int check_tree(int dtype, int32_t B, int32_t N, int32_t V) {
  if (dtype != TSD_F32 && dtype != TSD_BF16) return fail_no_handle(TSD_E_INVALID_ARG, "dtype must be TSD_F32 or TSD_BF16");
  if (B < 1 || N < 1 || V < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1, N >= 1, V >= 1");
  if (N > kTreeNodes) return fail_no_handle(TSD_E_OUT_OF_RANGE, "a tree has at most 256 nodes");
  if (V > kMostWords) return fail_no_handle(TSD_E_OUT_OF_RANGE, "V beyond 2^21");
  if (B > max_workgroups(1024)) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B beyond what a launch takes");
  return TSD_OK;
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_verify_tree_workspace(int32_t B, int32_t N, int32_t V, int32_t dtype, size_t* bytes_host) {
  const int rc = check_tree(dtype, B, N, V);
  if (rc) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  *bytes_host = 0;
  return TSD_OK;
}

extern "C" int tsd_verify_tree_static(const void* tokens_dev, const int32_t* parents_dev, int32_t parents_stride, const void* p_dev, int32_t dtype,
                                      int32_t token_bytes, int32_t B, int32_t N, int32_t V, int64_t p_stride_b, int64_t p_stride_n,
                                      const float* uniforms_dev, const void* choices_dev, const int32_t* n_new_dev, int32_t* n_acc_dev, void* out_dev,
                                      int32_t* path_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int rc = tsd_verify_tree_workspace(B, N, p_dev ? V : 1, p_dev ? dtype : TSD_F32, &need);
  if (rc) return rc;
  if (!tokens_dev || !parents_dev || !n_acc_dev || !out_dev || !path_dev)
    return fail_no_handle(TSD_E_INVALID_ARG, "tokens_dev, parents_dev, n_acc_dev, out_dev and path_dev must not be NULL");
  if (!p_dev == !choices_dev) return fail_no_handle(TSD_E_INVALID_ARG, "needs either p_dev or choices_dev");
  if (p_dev && !uniforms_dev) return fail_no_handle(TSD_E_INVALID_ARG, "uniforms_dev must not be NULL beside p_dev");
  if (token_bytes != 4 && token_bytes != 8) return fail_no_handle(TSD_E_INVALID_ARG, "token_bytes must be 4 or 8");
  if (parents_stride && parents_stride < N) return fail_no_handle(TSD_E_INVALID_ARG, "parents_stride must be 0 or at least N");
  if (p_dev && (p_stride_b < 0 || p_stride_n < 0)) return fail_no_handle(TSD_E_INVALID_ARG, "strides must not be negative");
  if (need && (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 7)))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that tsd_verify_tree_workspace gives for these sizes, 8-byte aligned");
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
  a.wide = token_bytes == 8;
  a.segments = p_dev ? (int)((V + (int64_t)kSegment - 1) / kSegment) : 0;
  const hipStream_t st = (hipStream_t)stream;
  const size_t lds = (size_t)a.segments * 16;
  if (!p_dev)
    verify_tree_kernel<void, 1><<<B, 64, lds, st>>>(a);
  else if (dtype == TSD_BF16)
    verify_tree_kernel<bf16, 16><<<B, 1024, lds, st>>>(a);
  else
    verify_tree_kernel<float, 16><<<B, 1024, lds, st>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("tree verification launch: ") + hipGetErrorString(e));
}
