// tsd_verify_tokens_static: drafted tokens against the target's probabilities, and the token drawn behind the last one that passed.
//
// Draft i (token x) of a sequence passes iff u_i q_i(x) < p_i(x); both sides are exact in 64 bits.  With n leading passes the next token is drawn
// from w = max(p_n - q_n, 0) where a draft failed, else from w = p_n: the first v with w_0 + .. + w_v > u_K W, W the sum of all.  The sums are
// held in 64 bits: over 10^5 fp32 terms a running sum in 32 would move one draw in a hundred to a neighbour.
//
// Memory bound: one row of p, and one of q where a draft failed.  A row goes in segments of kSegment elements, summed by a wavefront each; then the
// segment that crosses u_K W is found, and the token inside it.  Short rows, and those of many sequences, take one workgroup each; else a
// row's segments are dealt to several (some 512 in all), and the one that comes last goes on (last_arriver.h).  Rows start anywhere (an
// odd vocabulary), so 16-byte loads need no alignment beyond the element's.
// Three dependent trips to memory (drafts, their probabilities, the rows), 3 us, bound small calls: 1 x 4 drafts, 32000 fp32 probabilities
// 7.3 us; 64 x 6, 131072 fp32 16.4 us (58 MB: 3.5 TB/s); 256 x 8, 50257 bf16 14.0 us (41 MB: 2.9 TB/s).
#include <algorithm>

#include "draws.h"
#include "paged_cache.h"

namespace tsd {
namespace {

constexpr int kMaxDrafts = 16;
constexpr int kOneSegments = 256;  // most segments of a row that one workgroup sums

struct VerifyP {
  const void* draft;      // int32 or int64 [B][K]
  const void* q;          // NULL: every draft was certain
  const void* p;
  long p_sb, p_sr, q_sb, q_sr;
  const float* uniforms;  // [B][K + 1]
  const int* n_draft;
  int* n_acc;
  void* tokens;           // [B][K + 1]
  int B, K, V, wide;      // wide: 64-bit tokens
  int segments;
  int groups, per;        // workgroups that share a row, and the segments each of them takes
  double* sums;           // [2][B][segments]: of the row's weights, and of p alone where none of those is left
  uint64_t* slots;        // [B][groups]
  uint64_t tag;
};

// What a sequence's drafts come to, the same in every lane of a wavefront: how many passed, and the token of the one that failed
// (kNoToken: none of this vocabulary; kNoneFailed: all passed).
constexpr int kNoneFailed = -2;
struct Verdict {
  int n, failed;
};

template <typename T>
__device__ __forceinline__ Verdict test_drafts(const VerifyP& a, int b) {
  const int lane = threadIdx.x & 63;
  const int drafted = a.n_draft ? min(max(a.n_draft[b], 0), a.K) : a.K;
  bool pass = false;
  long x = -1;
  if (lane < drafted) {
    x = token_at(a.draft, (long)b * a.K + lane, a.wide);
    if (x >= 0 && x < a.V) {
      const double p = (double)(float)reinterpret_cast<const T*>(a.p)[b * a.p_sb + lane * a.p_sr + x];
      const double q = a.q ? (double)(float)reinterpret_cast<const T*>(a.q)[b * a.q_sb + lane * a.q_sr + x] : 1.0;
      pass = (double)a.uniforms[(long)b * (a.K + 1) + lane] * q < p;
    }
  }
  Verdict v;
  v.n = __builtin_ctzll(~__ballot(pass));  // (lanes from `drafted` on do not pass)
  v.failed = v.n == drafted ? kNoneFailed : __shfl(x >= 0 && x < a.V ? (int)x : kNoToken, v.n);
  return v;
}

template <typename T>
__device__ __forceinline__ Weights<T> weights_of(const VerifyP& a, int b, const Verdict& v) {
  Weights<T> w;
  w.p = reinterpret_cast<const T*>(a.p) + b * a.p_sb + v.n * a.p_sr;
  const bool failed = v.failed != kNoneFailed;
  w.q = failed && a.q ? reinterpret_cast<const T*>(a.q) + b * a.q_sb + v.n * a.q_sr : nullptr;
  w.without = failed && !a.q ? v.failed : kNoToken;
  return w;
}

// ONE: a workgroup sums a whole row, into LDS.  Else a row's workgroups sum `per` segments each, and the last of them draws.
template <typename T, int WAVES, bool ONE>
__global__ __launch_bounds__(WAVES * 64) void verify_kernel(const VerifyP a) {
  __shared__ double own_sums[ONE ? kOneSegments : 1];
  const int b = ONE ? blockIdx.x : blockIdx.x / a.groups, group = ONE ? 0 : blockIdx.x - b * a.groups;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double* sums = ONE ? own_sums : a.sums + (long)b * a.segments;
  const double u = (double)a.uniforms[(long)b * (a.K + 1) + a.K];
  const Verdict v = test_drafts<T>(a, b);
  Weights<T> w = weights_of<T>(a, b, v);
  for (int s = group * a.per + wave, end = ONE ? a.segments : min(a.segments, (group + 1) * a.per); s < end; s += WAVES) {
    const double sum = segment_sum(w, s, a.V);
    if (lane == 0) ONE ? (void)(sums[s] = sum) : leave(sums + s, sum);
  }
  if (ONE) {
    __syncthreads();
  } else {
    if (!came_last(a.slots + (long)b * a.groups, a.groups, group, a.tag)) return;
  }
  Found f = find_segment<ONE>(sums, a.segments, u);
  if (f.segment < 0 && (w.q || w.without >= 0)) {  // nothing is left of p over q: the draw goes by p (the same in every wavefront)
    w.q = nullptr;
    w.without = kNoToken;
    __syncthreads();
    if (!ONE) sums += (long)a.B * a.segments;  // (another finisher may still be reading the others)
    for (int s = wave; s < a.segments; s += WAVES) {
      const double sum = segment_sum(w, s, a.V);
      if (lane == 0) ONE ? (void)(sums[s] = sum) : leave(sums + s, sum);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    f = find_segment<ONE>(sums, a.segments, u);
  }
  if (!ONE) clear_slots(a.slots + (long)b * a.groups, a.groups);
  if (wave) return;
  const long token = f.segment < 0 ? -1 : find_token(w, f, a.V);
  if (lane <= a.K) {
    const long i = (long)b * (a.K + 1) + lane;
    const long x = lane < v.n ? token_at(a.draft, (long)b * a.K + lane, a.wide) : lane == v.n ? token : -1;
    if (a.wide)
      reinterpret_cast<long*>(a.tokens)[i] = x;
    else
      reinterpret_cast<int*>(a.tokens)[i] = (int)x;
  }
  if (lane == 0) a.n_acc[b] = v.n;
}

int check_verify(int dtype, int32_t B, int32_t K, int32_t V) {
  if (dtype != TSD_F32 && dtype != TSD_BF16) return fail_no_handle(TSD_E_INVALID_ARG, "dtype must be TSD_F32 or TSD_BF16");
  if (B < 1 || K < 1 || V < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1, K >= 1, V >= 1");
  if (K > kMaxDrafts) return fail_no_handle(TSD_E_OUT_OF_RANGE, "at most 16 drafts");
  if (B > max_workgroups(1024) || (int64_t)B * (V / kSegment + 4) > INT32_MAX) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B, or B * V, beyond what a launch takes");
  return TSD_OK;
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_verify_tokens_workspace(int32_t B, int32_t K, int32_t V, int32_t dtype, size_t* bytes_host) {
  const int rc = check_verify(dtype, B, K, V);
  if (rc) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  const size_t segments = (V + (size_t)kSegment - 1) / kSegment;
  *bytes_host = ((size_t)B * (2 * segments + (segments + 3) / 4) * 8 + 255) / 256 * 256;
  return TSD_OK;
}

extern "C" int tsd_verify_tokens_static(const void* draft_dev, const void* q_dev, const void* p_dev, int32_t dtype, int32_t token_bytes, int32_t B,
                                        int32_t K, int32_t V, int64_t q_stride_b, int64_t q_stride_k, int64_t p_stride_b, int64_t p_stride_k,
                                        const float* uniforms_dev, const int32_t* n_draft_dev, int32_t* n_acc_dev, void* tokens_dev,
                                        void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int rc = tsd_verify_tokens_workspace(B, K, V, dtype, &need);
  if (rc) return rc;
  if (!draft_dev || !p_dev || !uniforms_dev || !n_acc_dev || !tokens_dev)
    return fail_no_handle(TSD_E_INVALID_ARG, "draft_dev, p_dev, uniforms_dev, n_acc_dev and tokens_dev must not be NULL");
  if (token_bytes != 4 && token_bytes != 8) return fail_no_handle(TSD_E_INVALID_ARG, "token_bytes must be 4 or 8");
  if (q_stride_b < 0 || q_stride_k < 0 || p_stride_b < 0 || p_stride_k < 0) return fail_no_handle(TSD_E_INVALID_ARG, "strides must not be negative");
  if (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 7))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that tsd_verify_tokens_workspace gives for these sizes, 8-byte aligned");
  VerifyP a;
  a.draft = draft_dev;
  a.q = q_dev;
  a.p = p_dev;
  a.p_sb = p_stride_b;
  a.p_sr = p_stride_k;
  a.q_sb = q_stride_b;
  a.q_sr = q_stride_k;
  a.uniforms = uniforms_dev;
  a.n_draft = n_draft_dev;
  a.n_acc = n_acc_dev;
  a.tokens = tokens_dev;
  a.B = B;
  a.K = K;
  a.V = V;
  a.wide = token_bytes == 8;
  a.segments = (int)((V + (int64_t)kSegment - 1) / kSegment);
  a.sums = static_cast<double*>(workspace_dev);
  // (some 512 workgroups in all: 64 x 131072 fp32 with 4, 8, 16, 32 a row 20.1, 16.8, 17.5, 21.6 us, 128 x 65536 15.6, 16.6, 20.0, 20.1)
  const int want = (int)std::min<int64_t>((a.segments + 3) / 4, std::max(1, 512 / B));
  a.per = ((a.segments + want - 1) / want + 3) / 4 * 4;
  a.groups = (a.segments + a.per - 1) / a.per;
  a.slots = reinterpret_cast<uint64_t*>(a.sums + 2 * (size_t)B * a.segments);
  const hipStream_t st = (hipStream_t)stream;
  // One workgroup a row, us against several (fp32): 8000 x 4 sequences 7.5 / 9.1, 32000 x 1 8.0 / 7.7, 32000 x 160 11.6 / 13.4,
  // 131072 x 1 15.1 / 8.2, 131072 x 128 30.0 / 29.6 and x 200 36.6 / 45.8.
  const bool one = a.segments <= 16 || (B >= 160 && a.segments <= kOneSegments);
  a.tag = new_tag();
  const auto go = [&](auto split, auto whole) {
    if (one)
      whole<<<B, 1024, 0, st>>>(a);
    else
      split<<<(unsigned)((int64_t)B * a.groups), 256, 0, st>>>(a);
  };
  if (dtype == TSD_BF16)
    go(verify_kernel<bf16, 4, false>, verify_kernel<bf16, 16, true>);
  else
    go(verify_kernel<float, 4, false>, verify_kernel<float, 16, true>);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("token verification launch: ") + hipGetErrorString(e));
}
