// tsd_paged_attn_static on fp32 caches: as on bf16 ones, with the fp32 matrix instruction (16x16x4).  Its contraction is 4 deep and a lane holds one
// element of it, lane group g the g-th, so that both operands load as they lie:
//   S^T = K Q^T   lane group g takes 4 consecutive dims in one load, one per instruction (which dims an instruction contracts is free);
//                 lane (q, g) ends up with keys 4g .. 4g + 3 of each 16 for row q: the A operand of the next product, a key per instruction;
//   O += P V      lane (i, g) holds dims 4i .. 4i + 3 of every 64 of its key's row, one per instruction: no transposition.
// One token of 64 sequences of 2000 keys, 32 heads over 8 of 128: 185 us, 5.7 TB/s; 16 over 4 of 256: 188 us, 5.6.  2 x 1024 tokens behind 2048, 32 heads
// over 8 of 128: 934 us, 92 of the 148 TFLOP/s that a large product reaches: keys and values are fetched for every 32 rows; 16 over 4 of 256, where
// registers spill (64 bytes of scratch a lane, 136 below 256 dims): 1051 us, 82.  Short calls are bound by the matrix instructions of a step, 128 of
// 32 clocks for 80 dims as for 128, and three trips to memory.
#include "paged_attn.h"

namespace tsd {
namespace {

template <int DP, int MT, bool FULL>  // FULL: head_dim is DP
__global__ __launch_bounds__(kAttnWaves * 64, DP <= 64 ? 2 : 1) void paged_attn_f32_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KC = DP / 16, NC = DP / 64;
  AttnWork w = attn_place(p, 16 * MT);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int qi = lane & 15, g = lane >> 4;
  const int* table = p.cache.table + (long)w.b * p.cache.table_stride;
  const int stride = 32 * waves;
  int sb = w.key0 + 32 * wave;
  // (lane i and lane i + 32: key i of a step)
  int entry = paged_entry(p.cache, table, sb + (lane & 31)), next_entry = paged_entry(p.cache, table, sb + stride + (lane & 31));
  attn_lengths(p, w, 16 * MT);
  if (w.idle) return;
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
    for (int c = 0; c < KC; ++c) qf[mt][c] = FULL || c * 16 + g * 4 < p.D ? *reinterpret_cast<const f32x4*>(q + c * 16 + g * 4) : zero;
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
      for (int c = 0; c < KC; ++c) {
        const int d = c * 16 + g * 4;
        kf[bi][c] = *reinterpret_cast<const f32x4*>(k + (FULL || d < p.D ? d : 0));
        if (!FULL && d >= p.D) kf[bi][c] = zero;
      }
    }
  };
  auto load_v = [&](long off) {
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float* v = vbase + __shfl(off, 16 * bi + 4 * g + r);
#pragma unroll
        for (int c = 0; c < NC; ++c) vf[bi][r][c] = *reinterpret_cast<const f32x4*>(v + (FULL || c * 64 + qi * 4 < p.D ? c * 64 + qi * 4 : 0));  // (dims from D on: anything, never written)
      }
  };

  long off = attn_key_row(p, w, entry, sb + (lane & 31));
  entry = next_entry;
  unsigned valid = (unsigned)__ballot(off >= 0), next_valid = 0;
  if (sb < w.key1) {
    off = max(off, 0l);
    load_k(off);
    load_v(off);
  }
  off = attn_key_row(p, w, entry, sb + stride + (lane & 31));
  entry = paged_entry(p.cache, table, sb + 2 * stride + (lane & 31));
  bool odd = false;
  for (; sb < w.key1; sb += stride, valid = next_valid) {
    const bool more = sb + stride < w.key1;
    next_valid = (unsigned)__ballot(off >= 0);
    off = max(off, 0l);
    // (the entries of the step after the next are read before loads are issued that nothing waits for yet: counted waits do not
    // survive the branches between)
    const long later = attn_key_row(p, w, entry, sb + 2 * stride + (lane & 31));
    entry = paged_entry(p.cache, table, sb + 3 * stride + (lane & 31));
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
    if (!whole) {
      const bool mixed = w.see_first < w.see_last && sb + 32 > w.see_first;  // (see attn_take_out)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (!(valid >> (16 * bi + 4 * g + r) & 1)) vf[bi][r][c] = zero;
            if (mixed) odd |= attn_take_out(vf[bi][r][c]);
          }
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
    if (more) load_v(off);
    off = later;
  }

  if (__any(odd)) {
    for (int key = attn_mixed_from(w, 32); key < w.key1; ++key) {
      const long at = attn_key_row(p, w, paged_entry(p.cache, table, key), key);
      if (at < 0 || (key - w.key0) / 32 % waves != wave) continue;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const f32x4 x = FULL || c * 64 + qi * 4 < p.D ? *reinterpret_cast<const f32x4*>(vbase + at + c * 64 + qi * 4) : zero;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (key < __shfl(sees[mt], 4 * g + r)) o[mt][c][j][r] += attn_taken(x[j]);
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
  if (p.slots) attn_finish<float>(p, w, 16 * MT, reinterpret_cast<float*>(smem));
}

template <int DP>
hipError_t launch_dp(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const size_t lds = (size_t)waves * 16 * ((DP + 4) * 4 + 8);
  const auto go = [&](auto kernel) { kernel<<<grid, waves * 64, lds, st>>>(p); };
  if (mt == 1)
    go(p.D == DP ? paged_attn_f32_kernel<DP, 1, true> : paged_attn_f32_kernel<DP, 1, false>);
  else if constexpr (DP <= 128)
    go(p.D == DP ? paged_attn_f32_kernel<DP, 2, true> : paged_attn_f32_kernel<DP, 2, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn_f32(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  if (p.D <= 64) return launch_dp<64>(p, mt, waves, st);
  if (p.D <= 128) return launch_dp<128>(p, mt, waves, st);
  return launch_dp<256>(p, mt, waves, st);
}

}  // namespace tsd
