// tsd_paged_attn_static on bf16 caches, the join of split sequences, and the entry points.
//
// One wavefront takes 32 keys a step for 16 * MT rows:
//   S^T = K Q^T   two 16x16x32 MFMAs per 32 dims and row tile; key rows are permuted so that lane group g = lane / 16 ends up with the
//                 scores of the 8 consecutive keys 8g .. 8g + 7 for row lane % 16, which is the A operand of the next product;
//   online softmax in fp32, base 2 (running maximum and sum per row, shared by its 4 lanes).  The weights are rounded to bf16, the matrix
//                 instruction's operand, and the sum is that of the rounded ones: a weight's error of 2^-9 then moves the result only by
//                 the share of its value's distance from the mean;
//   O += P V      V rows are fetched with 16-byte loads, parked in LDS and picked up transposed with ds_read_b64_tr_b16.
// Few rows are memory bound: the next step's keys and values are asked for before this one's softmax, into the registers that its own
// left.
#include <algorithm>
#include <cmath>

#include "paged_attn.h"

namespace tsd {
namespace {

constexpr int v_stride(int dp) { return dp + 16; }  // V row in LDS: 32 bytes more than its dims, so that 8 rows fall on different banks

template <int DP, int MT>
__global__ __launch_bounds__(kAttnWaves * 64) void paged_attn_bf16_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KK = DP / 32, NB = DP / 16, VS = v_stride(DP), NV = DP / 16, VC = DP / 8;
  const AttnWork w = attn_work<16 * MT>(p);
  if (w.idle) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int qi = lane & 15, g = lane >> 4;
  const int* table = p.cache.table + (long)w.b * p.cache.table_stride;
  const bf16* kbase = reinterpret_cast<const bf16*>(p.cache.k) + w.hk * p.cache.head_stride;
  const bf16* vbase = reinterpret_cast<const bf16*>(p.cache.v) + w.hk * p.cache.head_stride;
  bf16* vt = reinterpret_cast<bf16*>(smem) + wave * 32 * VS;
  const bf16x8 zero = {};

  bf16x8 qf[MT][KK];
  int sees[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = w.row0 + mt * 16 + qi;
    sees[mt] = attn_sees(p, w, row);
    const int r = min(row, w.rows - 1), t = r / p.G, h = w.hk * p.G + r - t * p.G;
    const bf16* q = reinterpret_cast<const bf16*>(p.q.p) + w.b * p.q.sb + t * p.q.st + h * p.q.sh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = kk * 32 + g * 8;
      qf[mt][kk] = d < p.D ? *reinterpret_cast<const bf16x8*>(q + d) : zero;
    }
  }
  f32x4 o[MT][NB];
  float m_run[MT], l_run[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = -INFINITY;
    l_run[mt] = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[mt][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  auto lds_order = [] {  // orders this wavefront's own LDS traffic, which the hardware runs in issue order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  bf16x8 kf[2][KK], vf[NV];
  // (lane i and lane i + 32 hold the offset of key i of the step; where there is no key a lane reads row 0 of the pool, which always exists,
  // and what comes of it is dropped below)
  auto load_k = [&](long off) {
#pragma unroll
    for (int bi = 0; bi < 2; ++bi) {
      const bf16* k = kbase + __shfl(off, 8 * (qi >> 2) + 4 * bi + (qi & 3));
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int d = kk * 32 + g * 8;
        kf[bi][kk] = d < p.D ? *reinterpret_cast<const bf16x8*>(k + d) : zero;
      }
    }
  };
  auto load_v = [&](long off) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * 64 + lane, r = c / VC, d = (c - r * VC) * 8;
      const bf16* v = vbase + __shfl(off, r);
      vf[i] = d < p.D ? *reinterpret_cast<const bf16x8*>(v + d) : zero;
    }
  };

  const int stride = 32 * waves;
  int sb = w.key0 + 32 * wave;
  long off = attn_key_row(p, w, table, sb + (lane & 31));
  unsigned valid = (unsigned)__ballot(off >= 0), next_valid = 0;
  if (sb < w.key1) {
    off = max(off, 0l);
    load_k(off);
    load_v(off);
  }
  off = attn_key_row(p, w, table, sb + stride + (lane & 31));
  for (; sb < w.key1; sb += stride, valid = next_valid) {
    const bool more = sb + stride < w.key1;
    next_valid = (unsigned)__ballot(off >= 0);
    off = max(off, 0l);
    const bool whole = valid == 0xFFFFFFFFu && sb + 32 <= w.see_first;  // every row of the tile sees every key
    bool careful = false;
    if (!whole) {
      // keys that are not there hold anything; their weights are 0, and so must the values be
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (!(valid >> ((i * 64 + lane) / VC) & 1)) vf[i] = zero;
      // a value that is not finite, at a key that only some rows see, must not reach the others through 0 * inf
      if (w.see_first < w.see_last) {
        typedef unsigned uint4v __attribute__((ext_vector_type(4)));
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const uint4v x = __builtin_bit_cast(uint4v, vf[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) odd |= (x[j] & 0x7F80u) == 0x7F80u || (x[j] & 0x7F800000u) == 0x7F800000u;
        }
        careful = __any(odd);
      }
    }
    lds_order();  // the former step's reads before these writes
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * 64 + lane, r = c / VC;
      *reinterpret_cast<bf16x8*>(vt + r * VS + (c - r * VC) * 8) = vf[i];
    }
    lds_order();
    if (more) load_v(off);
    f32x4 sc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        sc[mt][bi] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) sc[mt][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[bi][kk], qf[mt][kk], sc[mt][bi], 0, 0, 0);
      }
    if (more) load_k(off);
    off = attn_key_row(p, w, table, sb + 2 * stride + (lane & 31));

    bf16x8 pf[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float s[8], e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = sc[mt][j >> 2][j & 3] * p.scale2;
      if (!whole) {
        const unsigned live = valid >> (8 * g);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!(live >> j & 1) || sb + 8 * g + j >= sees[mt]) s[j] = -INFINITY;
      }
      const float alpha = attn_running_max(s, m_run[mt], e);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pf[mt][j] = (bf16)e[j];
        sum += (float)pf[mt][j];
      }
      l_run[mt] = l_run[mt] * alpha + sum;
      if (__any(alpha != 1.f)) {  // accumulator rows are 4g + r: their factors come from those lanes
        float ar[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) ar[r] = __shfl(alpha, 4 * g + r);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[mt][nb][r] *= ar[r];
      }
    }
    auto values = [&](int nb) {  // the B operand of 16 dims
      typedef short short4v __attribute__((ext_vector_type(4)));
      short4v hv[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16* src = vt + (8 * g + 4 * half + (qi >> 2)) * VS + nb * 16 + 4 * (qi & 3);
        hv[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)src);
      }
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(hv[0], hv[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    if (!careful) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const bf16x8 vv = values(nb);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[mt], vv, o[mt][nb], 0, 0, 0);
      }
    } else {
      // key by key, added only to the rows that see it
#pragma unroll 1
      for (int key = 0; key < 32; ++key) {
        if (!(valid >> key & 1)) continue;
        const int j = key - 8 * g;  // (the lane's element that is this key, if it has it)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          bf16x8 pk = zero;
          int sees_it[4];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i == j) pk[i] = pf[mt][i];
#pragma unroll
          for (int r = 0; r < 4; ++r) sees_it[r] = sb + key < __shfl(sees[mt], 4 * g + r);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            bf16x8 vk = values(nb);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (i != j) vk[i] = (bf16)0.f;
            const f32x4 add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pk, vk, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (sees_it[r]) o[mt][nb][r] += add[r];
          }
        }
      }
    }
  }

  float* buf = reinterpret_cast<float*>(smem);
  float2* ml = reinterpret_cast<float2*>(buf + waves * 16 * (DP + 4));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float l = l_run[mt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    attn_join_tile<bf16, DP>(p, w, w.row0 + mt * 16, m_run[mt], l, buf, ml, [&](float* to, int rs) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[(4 * g + r) * rs + nb * 16 + qi] = o[mt][nb][r];
    });
  }
}

// A workgroup joins the chunks of one row: lanes take 4 dims, groups of lanes every so many chunks.
template <typename T>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(const PagedAttnP p) {
  __shared__ float part[256 * 5];
  const int h = blockIdx.x % p.Hq, bt = blockIdx.x / p.Hq, t = bt % p.T, b = bt / p.T;
  if (t >= attn_new(p, b)) return;
  const int chunks = attn_chunks(p, attn_len(p, b));
  const int lpr = p.D / 4, groups = 256 / lpr, d = (threadIdx.x % lpr) * 4, grp = threadIdx.x / lpr;
  const long row = ((long)b * p.splits * p.T + t) * p.Hq + h, step = (long)p.T * p.Hq;  // of chunk 0, and between chunks
  float mm = -INFINITY;
  for (int s = 0; s < chunks; ++s) mm = fmaxf(mm, p.part_lse[row + s * step]);
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (grp < groups)
    for (int s = grp; s < chunks; s += groups) {
      const float l = p.part_lse[row + s * step];
      if (l == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(l - mm);
      const f32x4 y = *reinterpret_cast<const f32x4*>(p.part_o + (row + s * step) * p.D + d);
      sum += f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * y[j];
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[threadIdx.x * 5 + j] = o[j];
  part[threadIdx.x * 5 + 4] = sum;
  __syncthreads();
  if (grp) return;
  for (int i = 1; i < groups; ++i) {
    const float* x = part + (threadIdx.x + i * lpr) * 5;
    sum += x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += x[j];
  }
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = (T)(o[j] * inv);
  *reinterpret_cast<T4*>(reinterpret_cast<T*>(p.out.p) + b * p.out.sb + t * p.out.st + h * p.out.sh + d) = y;
  if (d == 0 && p.lse) p.lse[((long)b * p.T + t) * p.Hq + h] = none ? -INFINITY : (mm + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

template <int DP>
hipError_t launch_dp(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const size_t stage = (size_t)waves * 32 * v_stride(DP) * 2, join = (size_t)waves * 16 * ((DP + 4) * 4 + 8);
  const size_t lds = stage > join ? stage : join;
  if (mt == 1)
    paged_attn_bf16_kernel<DP, 1><<<grid, waves * 64, lds, st>>>(p);
  else if (mt == 2)
    paged_attn_bf16_kernel<DP, 2><<<grid, waves * 64, lds, st>>>(p);
  else if constexpr (DP <= 128)
    paged_attn_bf16_kernel<DP, 4><<<grid, waves * 64, lds, st>>>(p);
  return hipGetLastError();
}

// What the sizes make of a call.
struct AttnPlan {
  int mt, waves, row_tiles, splits, chunk;
};

AttnPlan attn_plan(int dtype, int B, int T, int Hq, int Hkv, int D, int max_len) {
  AttnPlan a;
  const int rows = T * (Hq / Hkv);
  a.mt = rows <= 16 ? 1 : 2;
  a.row_tiles = (rows + 16 * a.mt - 1) / (16 * a.mt);
  a.waves = D > 128 ? 2 : max_len <= 128 ? 1 : kAttnWaves;
  const int64_t base = (int64_t)B * Hkv * a.row_tiles;
  const int64_t want = std::max<int64_t>(1, 1024 / base), most = std::max(1, max_len / 256);
  const int step = 32 * a.waves;
  const int64_t splits = std::min(want, most);
  a.chunk = (int)(((max_len + splits - 1) / splits + step - 1) / step * step);
  a.splits = (max_len + a.chunk - 1) / a.chunk;
  return a;
}

int check_attn(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len) {
  if (B < 1 || T < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1 and T >= 1");
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % cache->n_kv_heads)
    return fail_no_handle(TSD_E_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 1024");
  if (max_len < 1 || max_len > (1 << 30)) return fail_no_handle(TSD_E_INVALID_ARG, "max_len must be 1..2^30");
  if ((int64_t)B * T * n_q_heads > INT32_MAX) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B * T * n_q_heads beyond 2^31 - 1");
  return TSD_OK;
}

size_t attn_bytes(const AttnPlan& a, int B, int T, int Hq, int D) {
  if (a.splits == 1) return 0;
  const size_t rows = (size_t)B * a.splits * T * Hq;
  return (rows * D * 4 + rows * 4 + 255) / 256 * 256;
}

}  // namespace

hipError_t launch_paged_attn_bf16(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  if (p.D <= 64) return launch_dp<64>(p, mt, waves, st);
  if (p.D <= 96) return launch_dp<96>(p, mt, waves, st);
  if (p.D <= 128) return launch_dp<128>(p, mt, waves, st);
  return launch_dp<256>(p, mt, waves, st);
}

}  // namespace tsd

using namespace tsd;

extern "C" int tsd_paged_attn_workspace(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len, size_t* bytes_host) {
  const int rc = check_attn(cache, B, T, n_q_heads, max_len);
  if (rc) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  *bytes_host = attn_bytes(attn_plan(cache->dtype, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim, max_len), B, T, n_q_heads, cache->head_dim);
  return TSD_OK;
}

extern "C" int tsd_paged_attn_static(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* out,
                                     float* lse_dev, const int32_t* lens_dev, const int32_t* n_new_dev, int32_t max_len, float scale,
                                     void* workspace_dev, size_t workspace_bytes, void* stream) {
  int rc = check_attn(cache, B, T, n_q_heads, max_len);
  if (rc) return rc;
  const int es = type_bytes(cache->dtype);
  if ((rc = check_rows(q, es, "q")) || (rc = check_rows(out, es, "out"))) return rc;
  if (!lens_dev) return fail_no_handle(TSD_E_INVALID_ARG, "lens_dev must not be NULL");
  if (!std::isfinite(scale)) return fail_no_handle(TSD_E_INVALID_ARG, "scale must be finite");
  const AttnPlan a = attn_plan(cache->dtype, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim, max_len);
  const size_t need = attn_bytes(a, B, T, n_q_heads, cache->head_dim);
  if (need && (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that tsd_paged_attn_workspace gives for these sizes, 16-byte aligned");
  if ((int64_t)B * cache->n_kv_heads * a.row_tiles * a.splits > INT32_MAX) return fail_no_handle(TSD_E_OUT_OF_RANGE, "more than 2^31 workgroups");
  PagedAttnP p;
  p.cache = cache_view(*cache);
  p.q = rows_view(*q);
  p.out = rows_view(*out);
  p.lse = lse_dev;
  p.lens = lens_dev;
  p.n_new = n_new_dev;
  p.B = B;
  p.T = T;
  p.Hq = n_q_heads;
  p.Hkv = cache->n_kv_heads;
  p.G = n_q_heads / cache->n_kv_heads;
  p.D = cache->head_dim;
  p.row_tiles = a.row_tiles;
  p.splits = a.splits;
  p.chunk = a.chunk;
  p.scale2 = scale * 1.44269504088896341f;
  p.part_o = static_cast<float*>(workspace_dev);
  p.part_lse = need ? p.part_o + (size_t)B * a.splits * T * n_q_heads * cache->head_dim : nullptr;
  const hipStream_t st = (hipStream_t)stream;
  hipError_t e = cache->dtype == TSD_BF16 ? launch_paged_attn_bf16(p, a.mt, a.waves, st) : launch_paged_attn_f32(p, a.mt, a.waves, st);
  if (e == hipSuccess && a.splits > 1) {
    const unsigned rows = (unsigned)((int64_t)B * T * n_q_heads);
    if (cache->dtype == TSD_BF16)
      paged_attn_join_kernel<bf16><<<rows, 256, 0, st>>>(p);
    else
      paged_attn_join_kernel<float><<<rows, 256, 0, st>>>(p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("paged attention launch: ") + hipGetErrorString(e));
}
