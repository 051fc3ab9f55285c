// tsd_rope_append_static: rotary positions on the new tokens' queries and keys, and the keys and values written into a paged cache.
//
// A pair (a, b) of a head turns by angle = position * freq[i]: a' = a c - b s, b' = a s + b c.  The angle is formed in 64 bits and taken
// modulo one turn there (at position 100000 the fp32 product is off by 0.004 rad); sine and cosine of the rest, the rotation and its
// one rounding are fp32.
//
// Every element is read and written once, and nothing else is large: memory bound.  A workgroup takes one token, so that its R / 2 sines and cosines
// are formed once, in LDS, for all heads; its 16-byte items are the tokens' heads in a row (queries, keys, values).  16384 tokens of 32 + 8 + 8 heads
// of 128 in bf16: 72 us, 5.6 TB/s (a copy reaches 5.1).  One token: 2.5 us, a launch and two trips to memory.
#include <algorithm>
#include <cmath>

#include "paged_cache.h"

namespace tsd {
namespace {

struct RopeP {
  PagedView cache;
  RowsView q, q_out, k, v;
  const int* base;
  const int* n_new;
  const int* positions;
  const double* freq;
  int T, Hq, Hkv, D, R;
  float amplitude;
  int rot_items, copy_items;          // items of a rotated head and of a value head
  unsigned rot_magic, copy_magic;     // ceil(2^32 / items): n / items = (n * magic) >> 32 while n * items < 2^32; 0: one item
  int per_wg;                         // items a workgroup takes (a multiple of its lanes)
};

template <typename T>
struct Vec;
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  typedef bf16x8 V;
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  typedef f32x4 V;
};

// n / items by its magic (0: one item a head)
__device__ __forceinline__ int head_of(int n, unsigned magic) { return magic ? (int)__umulhi((unsigned)n, magic) : n; }

// WIDE: every item is 16 bytes (or a pair of them, one of each half); else single elements (R is no whole number of 16-byte items).
template <typename T, bool INTER, bool WIDE>
__global__ __launch_bounds__(256) void rope_append_kernel(const RopeP p) {
  constexpr int N = WIDE ? Vec<T>::N : 1;
  __shared__ float2 cs[128];
  const int b = blockIdx.x / p.T, t = blockIdx.x - b * p.T;
  if (p.n_new && t >= p.n_new[b]) return;
  const int slot = p.base[b] + t;
  const int pos = p.positions ? p.positions[blockIdx.x] : slot;
  for (int i = threadIdx.x; i < p.R / 2; i += 256) {
    const double turns = pos * p.freq[i] * 0.15915494309189533577;  // 1 / (2 pi)
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(p.amplitude * c, p.amplitude * s);
  }
  const long row = paged_row(p.cache, paged_entry(p.cache, p.cache.table + (long)b * p.cache.table_stride, slot), slot);
  __syncthreads();

  const int n_q = p.Hq * p.rot_items, n_rot = n_q + p.Hkv * p.rot_items, n_all = n_rot + p.Hkv * p.copy_items;
  const int first = blockIdx.y * p.per_wg, last = min(n_all, first + p.per_wg);
  for (int item = first + threadIdx.x; item < last; item += 256) {
    const T* src;
    T* dst;
    if (item < n_rot) {
      const int h = head_of(item, p.rot_magic), i = item - h * p.rot_items;
      if (h < p.Hq) {
        src = reinterpret_cast<const T*>(p.q.p) + b * p.q.sb + t * p.q.st + h * p.q.sh;
        dst = reinterpret_cast<T*>(p.q_out.p) + b * p.q_out.sb + t * p.q_out.st + h * p.q_out.sh;
      } else {
        if (row < 0) continue;
        src = reinterpret_cast<const T*>(p.k.p) + b * p.k.sb + t * p.k.st + (h - p.Hq) * p.k.sh;
        dst = reinterpret_cast<T*>(p.cache.k) + row + (h - p.Hq) * p.cache.head_stride;
      }
      const int pairs = p.R / 2;
      if constexpr (WIDE) {
        typedef typename Vec<T>::V V;
        const int turning = INTER ? p.R / N : pairs / N;  // items that turn; the rest copy
        if (i >= turning) {
          const int d = p.R + (i - turning) * N;
          *reinterpret_cast<V*>(dst + d) = *reinterpret_cast<const V*>(src + d);
        } else if constexpr (INTER) {
          V x = *reinterpret_cast<const V*>(src + i * N);
#pragma unroll
          for (int j = 0; j < N; j += 2) {
            const float2 w = cs[(i * N + j) / 2];
            const float a = (float)x[j], c = (float)x[j + 1];
            x[j] = (T)(a * w.x - c * w.y);
            x[j + 1] = (T)(a * w.y + c * w.x);
          }
          *reinterpret_cast<V*>(dst + i * N) = x;
        } else {
          V x = *reinterpret_cast<const V*>(src + i * N), y = *reinterpret_cast<const V*>(src + pairs + i * N);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const float2 w = cs[i * N + j];
            const float a = (float)x[j], c = (float)y[j];
            x[j] = (T)(a * w.x - c * w.y);
            y[j] = (T)(a * w.y + c * w.x);
          }
          *reinterpret_cast<V*>(dst + i * N) = x;
          *reinterpret_cast<V*>(dst + pairs + i * N) = y;
        }
      } else {
        if (i >= pairs) {
          dst[p.R + i - pairs] = src[p.R + i - pairs];
        } else {
          const int ia = INTER ? 2 * i : i, ib = INTER ? ia + 1 : i + pairs;
          const float2 w = cs[i];
          const float a = (float)src[ia], c = (float)src[ib];
          dst[ia] = (T)(a * w.x - c * w.y);
          dst[ib] = (T)(a * w.y + c * w.x);
        }
      }
    } else {
      if (row < 0) continue;
      const int m = item - n_rot, h = head_of(m, p.copy_magic), d = (m - h * p.copy_items) * Vec<T>::N;
      typedef typename Vec<T>::V V;
      *reinterpret_cast<V*>(reinterpret_cast<T*>(p.cache.v) + row + h * p.cache.head_stride + d) =
          *reinterpret_cast<const V*>(reinterpret_cast<const T*>(p.v.p) + b * p.v.sb + t * p.v.st + h * p.v.sh + d);
    }
  }
}

template <typename T>
hipError_t launch(const RopeP& p, bool inter, bool wide, dim3 grid, hipStream_t st) {
  if (inter && wide)
    rope_append_kernel<T, true, true><<<grid, 256, 0, st>>>(p);
  else if (inter)
    rope_append_kernel<T, true, false><<<grid, 256, 0, st>>>(p);
  else if (wide)
    rope_append_kernel<T, false, true><<<grid, 256, 0, st>>>(p);
  else
    rope_append_kernel<T, false, false><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_rope_append_static(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* q_out,
                                      const tsd_rows* k, const tsd_rows* v, const int32_t* base_dev, const int32_t* n_new_dev,
                                      const int32_t* positions_dev, const double* freq_dev, int32_t rotary_dim, float amplitude, uint32_t flags,
                                      void* stream) {
  if (B < 1 || T < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1 and T >= 1");
  int rc = check_cache(cache);
  if (rc) return rc;
  const int es = type_bytes(cache->dtype);
  if ((int64_t)B * T > max_workgroups(256)) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B * T beyond 2^24 - 1 tokens");
  if (n_q_heads < 1 || n_q_heads > 1024) return fail_no_handle(TSD_E_INVALID_ARG, "n_q_heads must be 1..1024");
  if ((rc = check_rows(q, es, "q")) || (rc = check_rows(q_out, es, "q_out")) || (rc = check_rows(k, es, "k")) || (rc = check_rows(v, es, "v"))) return rc;
  if (!base_dev || !freq_dev) return fail_no_handle(TSD_E_INVALID_ARG, "base_dev and freq_dev must not be NULL");
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > cache->head_dim) return fail_no_handle(TSD_E_INVALID_ARG, "rotary_dim must be even, 2..head_dim");
  if (!std::isfinite(amplitude)) return fail_no_handle(TSD_E_INVALID_ARG, "amplitude must be finite");
  if (flags & ~TSD_FLAG_ROPE_INTERLEAVED) return fail_no_handle(TSD_E_INVALID_ARG, "flags: only TSD_FLAG_ROPE_INTERLEAVED applies here");
  const bool inter = flags & TSD_FLAG_ROPE_INTERLEAVED;
  RopeP p;
  p.cache = cache_view(*cache);
  p.q = rows_view(*q);
  p.q_out = rows_view(*q_out);
  p.k = rows_view(*k);
  p.v = rows_view(*v);
  p.base = base_dev;
  p.n_new = n_new_dev;
  p.positions = positions_dev;
  p.freq = freq_dev;
  p.T = T;
  p.Hq = n_q_heads;
  p.Hkv = cache->n_kv_heads;
  p.D = cache->head_dim;
  p.R = rotary_dim;
  p.amplitude = amplitude;
  const int N = 16 / es;
  const bool wide = p.R % (inter ? N : 2 * N) == 0;
  p.rot_items = wide ? (inter ? p.R : p.R / 2) / N + (p.D - p.R) / N : p.R / 2 + (p.D - p.R);
  p.copy_items = p.D / N;
  const auto magic = [](int items) { return items > 1 ? (unsigned)((0x100000000ull + items - 1) / items) : 0u; };
  p.rot_magic = magic(p.rot_items);
  p.copy_magic = magic(p.copy_items);
  // Few tokens: their heads are dealt over several workgroups, as long as compute units are idle.
  const int64_t items = (int64_t)(p.Hq + p.Hkv) * p.rot_items + (int64_t)p.Hkv * p.copy_items;
  const int64_t turns = (items + 255) / 256, tokens = (int64_t)B * T;
  const int64_t parts = tokens >= 256 ? 1 : std::min<int64_t>(turns, (511 + tokens) / tokens);
  p.per_wg = (int)((turns + parts - 1) / parts) * 256;
  const dim3 grid((unsigned)tokens, (unsigned)((items + p.per_wg - 1) / p.per_wg));
  const hipError_t e = cache->dtype == TSD_BF16 ? launch<bf16>(p, inter, wide, grid, (hipStream_t)stream) : launch<float>(p, inter, wide, grid, (hipStream_t)stream);
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("rotary append launch: ") + hipGetErrorString(e));
}
