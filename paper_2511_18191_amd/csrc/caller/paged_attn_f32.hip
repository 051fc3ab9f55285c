// tsd_paged_attn_static on fp32 caches: as on bf16 ones, with the fp32 matrix instruction (16x16x4).  Its contraction is 4 deep and a lane holds one
// element of it, lane group g the g-th, so that both operands load as they lie:
//   S^T = K Q^T   lane group g takes 4 consecutive dims in one load, one per instruction (which dims an instruction contracts is free);
//                 lane (q, g) ends up with keys 4g .. 4g + 3 of each 16 for row q: the A operand of the next product, a key per instruction;
//   O += P V      lane (i, g) holds dims 4i .. 4i + 3 of every 64 of its key's row, one per instruction: no transposition.
#include "paged_attn.h"

namespace tsd {
namespace {

template <int DP, int MT>
__global__ __launch_bounds__(kAttnWaves * 64) void paged_attn_f32_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KC = DP / 16, NC = DP / 64;
  const AttnWork w = attn_work<16 * MT>(p);
  if (w.idle) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int qi = lane & 15, g = lane >> 4;
  const int* table = p.cache.table + (long)w.b * p.cache.table_stride;
  const float* kbase = reinterpret_cast<const float*>(p.cache.k) + w.hk * p.cache.head_stride;
  const float* vbase = reinterpret_cast<const float*>(p.cache.v) + w.hk * p.cache.head_stride;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

  f32x4 qf[MT][KC];
  int sees[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = w.row0 + mt * 16 + qi;
    sees[mt] = attn_sees(p, w, row);
    const int r = min(row, w.rows - 1), t = r / p.G, h = w.hk * p.G + r - t * p.G;
    const float* q = reinterpret_cast<const float*>(p.q.p) + w.b * p.q.sb + t * p.q.st + h * p.q.sh;
#pragma unroll
    for (int c = 0; c < KC; ++c) qf[mt][c] = c * 16 + g * 4 < p.D ? *reinterpret_cast<const f32x4*>(q + c * 16 + g * 4) : zero;
  }
  f32x4 o[MT][NC][4];  // [..][j]: dim 64 c + 4 qi + j of rows 4g ..
  float m_run[MT], l_run[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = -INFINITY;
    l_run[mt] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[mt][c][j] = zero;
  }

  f32x4 kf[2][KC], vf[2][4][NC];
  auto load_k = [&](long off) {
#pragma unroll
    for (int bi = 0; bi < 2; ++bi) {
      const float* k = kbase + __shfl(off, 16 * bi + qi);
#pragma unroll
      for (int c = 0; c < KC; ++c) kf[bi][c] = c * 16 + g * 4 < p.D ? *reinterpret_cast<const f32x4*>(k + c * 16 + g * 4) : zero;
    }
  };
  auto load_v = [&](long off) {
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float* v = vbase + __shfl(off, 16 * bi + 4 * g + r);
#pragma unroll
        for (int c = 0; c < NC; ++c) vf[bi][r][c] = c * 64 + qi * 4 < p.D ? *reinterpret_cast<const f32x4*>(v + c * 64 + qi * 4) : zero;
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
    const bool whole = valid == 0xFFFFFFFFu && sb + 32 <= w.see_first;
    f32x4 sc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        sc[mt][bi] = zero;
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[mt][bi] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[bi][c][j], qf[mt][c][j], sc[mt][bi], 0, 0, 0);
      }
    if (more) load_k(off);
    bool careful = false;
    if (!whole) {
      bool odd = false;
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (!(valid >> (16 * bi + 4 * g + r) & 1)) vf[bi][r][c] = zero;
#pragma unroll
            for (int j = 0; j < 4; ++j) odd |= (__float_as_uint(vf[bi][r][c][j]) & 0x7F800000u) == 0x7F800000u;
          }
      careful = w.see_first < w.see_last && __any(odd);
    }
    float e[MT][8];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float s[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[j] = sc[mt][j >> 2][j & 3] * p.scale2;
        const int key = 16 * (j >> 2) + 4 * g + (j & 3);
        if (!whole && (!(valid >> key & 1) || sb + key >= sees[mt])) s[j] = -INFINITY;
      }
      const float alpha = attn_running_max(s, m_run[mt], e[mt]);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += e[mt][j];
      l_run[mt] = l_run[mt] * alpha + sum;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float ar = __shfl(alpha, 4 * g + r);
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[mt][c][j][r] *= ar;
        }
      }
    }
    if (!careful) {
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
                o[mt][c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(e[mt][4 * bi + r], vf[bi][r][c][j], o[mt][c][j], 0, 0, 0);
    } else {
      // key by key, added only to the rows that see it: a value that is not finite must not reach the others through 0 * inf
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll 1
        for (int gg = 0; gg < 4; ++gg) {
          const int key = 16 * (x >> 2) + 4 * gg + (x & 3);
          if (!(valid >> key & 1)) continue;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            int sees_it[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) sees_it[r] = sb + key < __shfl(sees[mt], 4 * g + r);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const f32x4 add =
                    __builtin_amdgcn_mfma_f32_16x16x4f32(g == gg ? e[mt][x] : 0.f, g == gg ? vf[x >> 2][x & 3][c][j] : 0.f, zero, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (sees_it[r]) o[mt][c][j][r] += add[r];
              }
          }
        }
    }
    if (more) load_v(off);
    off = attn_key_row(p, w, table, sb + 2 * stride + (lane & 31));
  }

  float* buf = reinterpret_cast<float*>(smem);
  float2* ml = reinterpret_cast<float2*>(buf + waves * 16 * (DP + 4));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float l = l_run[mt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    attn_join_tile<float, DP>(p, w, w.row0 + mt * 16, m_run[mt], l, buf, ml, [&](float* to, int rs) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          f32x4 y;
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = o[mt][c][j][r];
          *reinterpret_cast<f32x4*>(to + (4 * g + r) * rs + c * 64 + qi * 4) = y;
        }
    });
  }
}

template <int DP>
hipError_t launch_dp(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const size_t lds = (size_t)waves * 16 * ((DP + 4) * 4 + 8);
  if (mt == 1)
    paged_attn_f32_kernel<DP, 1><<<grid, waves * 64, lds, st>>>(p);
  else if (mt == 2)
    paged_attn_f32_kernel<DP, 2><<<grid, waves * 64, lds, st>>>(p);
  else if constexpr (DP <= 128)
    paged_attn_f32_kernel<DP, 4><<<grid, waves * 64, lds, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn_f32(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  if (p.D <= 64) return launch_dp<64>(p, mt, waves, st);
  if (p.D <= 128) return launch_dp<128>(p, mt, waves, st);
  return launch_dp<256>(p, mt, waves, st);
}

}  // namespace tsd
