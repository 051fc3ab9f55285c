// tsd_paged_attn_static on fp32 caches: as on bf16 ones, with the fp32 matrix instruction (16x16x4).  Its contraction is 4 deep and a lane holds one
// element of it, lane group g the g-th, so that both operands load as they lie:
//   S^T = K Q^T   lane group g takes 4 consecutive dims in one load, one per instruction (which dims an instruction contracts is free);
//                 lane (q, g) ends up with keys 4g .. 4g + 3 of each 16 for row q: the A operand of the next product, a key per instruction;
//   O += P V      lane (i, g) holds dims 4i .. 4i + 3 of every 64 of its key's row, one per instruction: no transposition.
// One token of 64 sequences of 2000 keys, 32 heads over 8 of 128: 185 us, 5.7 TB/s; 16 over 4 of 256: 182 us, 5.8.  2 x 1024 tokens behind 2048, 32 heads
// over 8 of 128: 934 us, 92 of the 148 TFLOP/s that a large product reaches: keys and values are fetched for every 32 rows; 16 over 4 of 256: 1049 us, 82.
// Short calls are bound by the matrix instructions of a step, 104 of 32 clocks for 80 dims, 128 for 128, and three trips to memory; heads of 80 and 96 dims have kernels of their own, two wavefronts of which share a SIMD
// (12 heads over 4 of 80: 3 tokens of 6 sequences of up to 1501 keys, eight draws of lengths, 13.8 to 15.1 us in the one for 128 dims, 11.8 to 15.5 so, longer where one long sequence is
// what a draw waits for; 5 tokens of 24 sequences 34.8 and 29.6, one of 64 of up to 4000 keys 167 and 105;
// trees of up to 17 nodes of 24 such sequences at a window of 500 34).
#include "paged_attn.h"

namespace tsd {
namespace {

template <int M, int DP, int MT, bool FULL>  // M: AttnMask; FULL: head_dim is DP
__global__ __launch_bounds__(kAttnWaves * 64, DP <= 64 || (DP <= 96 && MT == 1) ? 2 : 1) void paged_attn_f32_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KC = DP / 16, NC = (DP + 63) / 64;
  constexpr bool kAll = FULL && NC * 64 == DP;  // every lane's dims of the values are there
  constexpr int kSure = FULL ? DP : DP == 64 ? 8 : DP == 80 ? 72 : DP == 96 ? 88 : DP == 128 ? 104 : 136;  // dims that every head of this kernel has
  AttnWork w = attn_place(p, 16 * MT);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int qi = lane & 15, g = lane >> 4;
  const int* table = p.cache.table + (long)w.b * p.cache.table_stride;
  const int stride = 32 * waves;
  int sb = w.key0 + 32 * wave;
  // (lane i and lane i + 32: key i of a step)
  // (the table's entries are on their way before the lengths are there: nearly always places are keys)
  int entry = paged_entry(p.cache, table, sb + (lane & 31)), next_entry = paged_entry(p.cache, table, sb + stride + (lane & 31));
  const AttnParents<M> parents(p, w);
  attn_lengths<M>(p, w, 16 * MT);
  if (w.idle) return;
  if (M != kCausal && w.gap) {
    entry = attn_entry<M>(p, w, table, sb + (lane & 31));
    next_entry = attn_entry<M>(p, w, table, sb + stride + (lane & 31));
  }
  __shared__ std::conditional_t<M == kTree, AttnLines, int> lines;
  if constexpr (M == kTree) attn_lines(p, w, parents, 16 * MT, lines);
  // (what a row sees; of nodes only where it is, in registers)
  const auto sight = [&](int row) {
    if constexpr (M == kTree)
      return attn_line_at(p, w, row);
    else
      return attn_sight<M>(p, w, row);
  };
  const auto seen = [&](auto by, int from) {
    if constexpr (M == kTree)
      return attn_seen<M>(p, w, attn_line_sight(p, w, lines, by), from);
    else
      return attn_seen<M>(p, w, by, from);
  };
  const float* kbase = reinterpret_cast<const float*>(p.cache.k) + w.hk * p.cache.head_stride;
  const float* vbase = reinterpret_cast<const float*>(p.cache.v) + w.hk * p.cache.head_stride;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

  // Above 128 dims the queries stay in LDS: with them registers spilled, and a value of four that the compiler keeps half in matrix registers and half in
  // memory came back without one of its parts (wrong scores; ROCm 7.2).
  constexpr bool kStaged = DP > 128;
  constexpr int QS = DP + 4;
  static_assert(!kStaged || MT == 1);
  float* staged = reinterpret_cast<float*>(smem);  // [16][QS], until the join takes the place
  f32x4 qf[MT][kStaged ? 1 : KC];
  decltype(sight(0)) sees[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = w.row0 + mt * 16 + qi;
    sees[mt] = sight(row);
    const int r = min(row, w.rows - 1), t = r / p.G, h = w.hk * p.G + r - t * p.G;
    const float* q = reinterpret_cast<const float*>(p.q.p) + w.b * p.q.sb + t * p.q.st + h * p.q.sh;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const f32x4 x = c * 16 + 16 <= kSure || c * 16 + g * 4 < p.D ? *reinterpret_cast<const f32x4*>(q + c * 16 + g * 4) : zero;
      if constexpr (!kStaged)
        qf[mt][c] = x;
      else if (wave == 0)
        *reinterpret_cast<f32x4*>(staged + qi * QS + c * 16 + g * 4) = x;
    }
  }
  if constexpr (kStaged) __syncthreads();
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
        const bool in = c * 16 + 16 <= kSure || d < p.D;
        kf[bi][c] = *reinterpret_cast<const f32x4*>(k + (in ? d : 0));
        if (!in) kf[bi][c] = zero;
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
        for (int c = 0; c < NC; ++c) vf[bi][r][c] = *reinterpret_cast<const f32x4*>(v + (kAll || c * 64 + qi * 4 < p.D ? c * 64 + qi * 4 : 0));  // (dims from D on: anything, never written)
      }
  };

  long off = attn_key_row<M>(p, w, entry, sb + (lane & 31));
  entry = next_entry;
  unsigned valid = (unsigned)__ballot(off >= 0), next_valid = 0;
  if (sb < w.key1) {
    off = max(off, 0l);
    load_k(off);
    load_v(off);
  }
  off = attn_key_row<M>(p, w, entry, sb + stride + (lane & 31));
  entry = attn_entry<M>(p, w, table, sb + 2 * stride + (lane & 31));
  bool odd = false;
  for (; sb < w.key1; sb += stride, valid = next_valid) {
    const bool more = sb + stride < w.key1;
    next_valid = (unsigned)__ballot(off >= 0);
    off = max(off, 0l);
    // (the entries of the step after the next are read before loads are issued that nothing waits for yet: counted waits do not
    // survive the branches between)
    const long later = attn_key_row<M>(p, w, entry, sb + 2 * stride + (lane & 31));
    entry = attn_entry<M>(p, w, table, sb + 3 * stride + (lane & 31));
    const bool whole = valid == 0xFFFFFFFFu && attn_all_see<M>(p, w, sb, 32);
    f32x4 sc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        sc[mt][bi] = zero;
        if constexpr (kStaged) asm volatile("" ::: "memory");  // (read anew in every step, not kept)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          f32x4 x;
          if constexpr (kStaged)
            x = *reinterpret_cast<const f32x4*>(staged + qi * QS + c * 16 + g * 4);
          else
            x = qf[mt][c];
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[mt][bi] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[bi][c][j], x[j], sc[mt][bi], 0, 0, 0);
        }
      }
    if (more) load_k(off);
    if (!whole) {
      const bool mixed = attn_mixed<M>(p, w, sb, 32);  // (see attn_take_out)
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
      unsigned live = valid;
      if constexpr (M != kCausal)
        if (!whole) live &= seen(sees[mt], sb);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[j] = sc[mt][j >> 2][j & 3] * p.scale2;
        const int key = 16 * (j >> 2) + 4 * g + (j & 3);
        // (a causal row's keys are compared: its bits, formed in every step, took one token of 64 sequences of up to 4000 keys, 12 heads over 4 of 64, from 59.7 us to 61.4)
        if constexpr (M == kCausal) {
          if (!whole && (!(live >> key & 1) || sb + key >= sees[mt].sees)) s[j] = -INFINITY;
        } else {
          if (!whole && !(live >> key & 1)) s[j] = -INFINITY;
        }
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
    for (int key = attn_mixed_from<M>(w, 32); key < w.key1; ++key) {
      const long at = attn_key_row<M>(p, w, attn_entry<M>(p, w, table, key), key);
      if (at < 0 || (key - w.key0) / 32 % waves != wave || (M != kCausal && !attn_mixed<M>(p, w, key - (key - w.key0) % 32, 32))) continue;
      unsigned reached = 0;  // (by the lane's rows)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (M == kCausal)
            reached |= key < __shfl(sees[mt].sees, 4 * g + r) ? 1u << (4 * mt + r) : 0u;
          else
            reached |= (seen(sight(w.row0 + mt * 16 + 4 * g + r), key) & 1) << (4 * mt + r);
        }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const f32x4 x = kAll || c * 64 + qi * 4 < p.D ? *reinterpret_cast<const f32x4*>(vbase + at + c * 64 + qi * 4) : zero;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (reached >> (4 * mt + r) & 1) o[mt][c][j][r] += attn_taken(x[j]);
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
          if (NC * 64 == DP || c * 64 + qi * 4 < DP) *reinterpret_cast<f32x4*>(to + (4 * g + r) * rs + c * 64 + qi * 4) = y;
        }
    });
  }
  if (p.slots) attn_finish<float>(p, w, 16 * MT, reinterpret_cast<float*>(smem));
}

template <int M, int DP>
hipError_t launch_dp(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const size_t lds = (size_t)waves * 16 * ((DP + 4) * 4 + 8);
  const auto go = [&](auto kernel) { kernel<<<grid, waves * 64, lds, st>>>(p); };
  if (mt == 1)
    go(p.D == DP ? paged_attn_f32_kernel<M, DP, 1, true> : paged_attn_f32_kernel<M, DP, 1, false>);
  else if constexpr (DP <= 128)
    go(p.D == DP ? paged_attn_f32_kernel<M, DP, 2, true> : paged_attn_f32_kernel<M, DP, 2, false>);
  return hipGetLastError();
}

template <int M>
hipError_t launch_mask(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  if (p.D <= 64) return launch_dp<M, 64>(p, mt, waves, st);
  if (p.D <= 80) return launch_dp<M, 80>(p, mt, waves, st);
  if (p.D <= 96) return launch_dp<M, 96>(p, mt, waves, st);
  if (p.D <= 128) return launch_dp<M, 128>(p, mt, waves, st);
  return launch_dp<M, 256>(p, mt, waves, st);
}

}  // namespace

hipError_t launch_paged_attn_f32(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  return p.mask == kCausal ? launch_mask<kCausal>(p, mt, waves, st) : p.mask == kWindow ? launch_mask<kWindow>(p, mt, waves, st) : launch_mask<kTree>(p, mt, waves, st);
}

}  // namespace tsd
