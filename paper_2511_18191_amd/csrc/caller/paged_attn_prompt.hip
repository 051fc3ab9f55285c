// tsd_paged_attn_static on bf16 caches, many rows: chunks of prompts.
//
// Operations bound these calls, so keys and values are staged in LDS once for all rows of a workgroup (32 a wavefront), and both products run on
// 32x32x16 matrix instructions with the rows along the lanes:
//   S^T = K Q^T    lane (row r = lane % 32, half h = lane / 32) ends up with keys 8 i + 4 h + j (i, j < 4) of each 32;
//   O^T += V^T P^T the contraction's order is free, so those same keys are its operand as they lie, and V rows are picked up transposed for
//                  them (ds_read_b64_tr_b16: 4 keys of one dim).
// Maximum, sum and rescaling of a row stay in its two lanes: one exchange between the halves per 64 keys, and nothing crosses lanes for the
// sums.  The weights are rounded to bf16, the instruction's operand, and the sum is that of the rounded ones, as in paged_attn.hip, by the dot product
// of two weights with ones (rounded once, to fp32).  The heaviest weight is 1 and exact: sums are rescaled by every key that is the largest
// so far.  Where the logarithm of the denominator is asked for, the unrounded weights are summed beside, and it (and the join of parts) is of these.
// (Sums relative to a maximum that lagged by up to 2^6, of unrounded weights, took 77 us for 81 with 2 x 1024 tokens over 2048 keys, 32 heads over 8 of
// 128, and 41 for 44 with 16 heads of 64, and were less exact: scores of deviation 1.5, 4, 8 were off by 2.21, 1.86, 1.73 in 1000 where this is by
// 1.92, 1.68, 1.64, and the result's rounding alone by 1.66, 1.67, 1.64.)
// 32 rows a wavefront at 252 registers, two on a SIMD: one forms weights while the other multiplies.  (64 rows would read LDS half as often, but
// do not fit: 350 registers and spills.)
// 2 x 1024 tokens behind 2048, 32 heads over 8 of 128: 125 us, 0.69 PFLOP/s; 16 heads of 64: 63 us, 0.34; weights and products overlap only in part, and
// both take some 1000 clocks per 64 keys and 32 rows of 128.
#include "paged_attn.h"

namespace tsd {
namespace {

constexpr int kTile = 64;  // keys a tile

// 16-byte chunk `c` of row `r` lies at chunk c ^ turn(r) of its row: one chunk of 16 rows, and four of 4, cover all 256 bytes of the banks.
template <int DP>
__device__ __forceinline__ int turn(int r) {
  return DP == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

template <int DP, int WAVES, bool FULL, bool LSE>  // FULL: head_dim is DP; LSE: the logarithms are asked for
__global__ __launch_bounds__(WAVES * 64, 2) void paged_attn_prompt_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int kWaveRows = 32, KK = DP / 16, DB = DP / 32, CPR = DP / 8, THREADS = WAVES * 64, NL = kTile * CPR / THREADS;
  AttnWork w = attn_place(p, WAVES * kWaveRows);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r32 = lane & 31, h = lane >> 5;
  const int* table = p.cache.table + (long)w.b * p.cache.table_stride;
  int entry = paged_entry(p.cache, table, w.key0 + lane), next_entry = paged_entry(p.cache, table, w.key0 + kTile + lane);
  attn_lengths(p, w, WAVES * kWaveRows);
  if (w.idle) return;
  const bf16* kbase = reinterpret_cast<const bf16*>(p.cache.k) + w.hk * p.cache.head_stride;
  const bf16* vbase = reinterpret_cast<const bf16*>(p.cache.v) + w.hk * p.cache.head_stride;
  bf16* lds = reinterpret_cast<bf16*>(smem);  // [2][K, V][kTile][DP]
  const bf16x8 zero = {};
  const float scale2 = fmaxf(fabsf(p.scale2), 1.2e-38f);

  const int row0 = w.row0 + wave * kWaveRows;
  const int row = row0 + r32, sees = attn_sees(p, w, row);
  bf16x8 qf[KK];
  {
    const int r = min(row, w.rows - 1), t = r / p.G, hq = w.hk * p.G + r - t * p.G;
    const bf16* q = reinterpret_cast<const bf16*>(p.q.p) + w.b * p.q.sb + t * p.q.st + hq * p.q.sh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = kk * 16 + h * 8;
      qf[kk] = FULL || d < p.D ? *reinterpret_cast<const bf16x8*>(q + d) : zero;
      if (p.scale2 < 0.f) qf[kk] = -qf[kk];
    }
  }
  // keys that the wavefront's first and last rows see (a wavefront without rows only loads)
  const int see_first = row0 + kWaveRows <= w.rows ? attn_sees(p, w, row0) : 0;
  const int see_last = row0 < w.rows ? attn_sees(p, w, min(row0 + kWaveRows, w.rows) - 1) : 0;

  f32x16 o[DB];
  float m_run = -INFINITY, l_run = 0.f, l_true = 0.f;  // (l_true: of the unrounded weights)
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

  bf16x8 kr[NL], vr[NL];
  auto load = [&](long off, unsigned long long there) {
    if (FULL && there == ~0ull) {  // (nearly always: no lane has to be kept from its load)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int c = i * THREADS + threadIdx.x;
        const long o_r = __shfl(off, c / CPR) + (c % CPR) * 8;
        kr[i] = *reinterpret_cast<const bf16x8*>(kbase + o_r);
        vr[i] = *reinterpret_cast<const bf16x8*>(vbase + o_r);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int c = i * THREADS + threadIdx.x, r = c / CPR, d = (c % CPR) * 8;
      const long o_r = __shfl(off, r);
      const bool in = o_r >= 0 && (FULL || d < p.D);
      kr[i] = in ? *reinterpret_cast<const bf16x8*>(kbase + o_r + d) : zero;
      vr[i] = in ? *reinterpret_cast<const bf16x8*>(vbase + o_r + d) : zero;
    }
  };
  long off = attn_key_row(p, w, entry, w.key0 + lane);
  entry = next_entry;
  unsigned long long valid = __ballot(off >= 0), next_valid = 0;
  if (w.key0 < w.key1) load(off, valid);
  off = attn_key_row(p, w, entry, w.key0 + kTile + lane);
  entry = paged_entry(p.cache, table, w.key0 + 2 * kTile + lane);
  int parity = 0;
  bool odd = false;
  for (int sb = w.key0; sb < w.key1; sb += kTile, valid = next_valid, parity ^= 1) {
    bf16* kt = lds + parity * 2 * kTile * DP;
    bf16* vt = kt + kTile * DP;
    next_valid = __ballot(off >= 0);
    const bool mixed = sb + kTile > w.see_first && w.see_first < w.see_last;  // (the same in every wavefront; see attn_take_out)
    if (mixed) {
#pragma unroll
      for (int i = 0; i < NL; ++i) odd |= attn_take_out(vr[i]);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int c = i * THREADS + threadIdx.x, r = c / CPR, at = r * DP + ((c % CPR) ^ turn<DP>(r)) * 8;
      *reinterpret_cast<bf16x8*>(kt + at) = kr[i];
      *reinterpret_cast<bf16x8*>(vt + at) = vr[i];
    }
    // (two buffers: who writes one has left it a barrier ago)
    __syncthreads();
    // (the entries of the tile after the next are read before loads are issued that nothing waits for yet: counted waits do not
    // survive the branches between)
    const long later = attn_key_row(p, w, entry, sb + 2 * kTile + lane);
    entry = paged_entry(p.cache, table, sb + 3 * kTile + lane);
    if (sb + kTile < w.key1) load(off, next_valid);
    off = later;
    if (sb >= see_last) continue;

    f32x16 sc[2];  // of 32 keys each
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[s][i] = 0.f;
      const int r = s * 32 + r32;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + r * DP + ((2 * kk + h) ^ turn<DP>(r)) * 8);
        sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], sc[s], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    const bool whole = valid == ~0ull && sb + kTile <= see_first;
    if (!whole) {
      const int left = sees - sb - 4 * h;  // (the lane's keys are 4 h further on than these)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const unsigned there = (unsigned)(valid >> (4 * h) >> (32 * s));
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!(there >> (8 * (i >> 2) + (i & 3)) & 1) || s * 32 + 8 * (i >> 2) + (i & 3) >= left) sc[s][i] = -INFINITY;
      }
    }
    // (maxima are those of the products; a negative factor has gone into the queries, and one of 0 is too small to tell scores apart)
    float mx = sc[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) mx = fmaxf(mx, sc[i >> 4][i & 15]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const bool raise = mx > m_run;  // (the first key a row sees, too)
    if (__any(raise)) {
      float alpha = 1.f;
      if (raise) {
        alpha = __builtin_amdgcn_exp2f((m_run - mx) * scale2);
        m_run = mx;
      }
      l_run *= alpha;
      if (LSE) l_true *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    const float shift = m_run == -INFINITY ? 0.f : -m_run * scale2;
    // 32 keys' weights, then their product with the values: the matrix cores run behind while the next weights are formed
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 pf[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(sc[s][i], scale2, shift));
        if (LSE) l_true += e;
        pf[i >> 3][i & 7] = (bf16)e;
      }
      typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 ones = {(bf16)1.f, (bf16)1.f};
#pragma unroll
      for (int i = 0; i < 16; i += 2) l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[i >> 3][i & 7], pf[i >> 3][(i & 7) + 1]}, ones, l_run, false);
      // operand of the values: keys 16 m + 8 (j / 4) + 4 h + j % 4, j = 0 .. 7, for dim lane % 32 of a block
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          typedef short short4v __attribute__((ext_vector_type(4)));
          short4v hv[2];
          const int l16 = lane & 15, half16 = (lane >> 4) & 1;
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const int r = s * 32 + m * 16 + part * 8 + h * 4 + (l16 >> 2), c = db * 4 + half16 * 2 + ((l16 & 3) >> 1);
            const bf16* src = vt + r * DP + (c ^ turn<DP>(r)) * 8 + (l16 & 1) * 4;
            hv[part] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)src);
          }
          const bf16x8 vv = __builtin_bit_cast(bf16x8, __builtin_shufflevector(hv[0], hv[1], 0, 1, 2, 3, 4, 5, 6, 7));
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, pf[m], o[db], 0, 0, 0);
        }
    }
  }
  if (__syncthreads_or(odd)) {
    for (int key = attn_mixed_from(w, kTile); key < w.key1; ++key) {
      const long at = attn_key_row(p, w, paged_entry(p.cache, table, key), key);
      if (at < 0) continue;
#pragma unroll
      for (int i = 0; i < DB * 4; ++i) {
        const int d = 8 * i + 4 * h;
        bf16x4 v = {};
        if (FULL || d < p.D) v = *reinterpret_cast<const bf16x4*>(vbase + at + d);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (key < sees) o[i >> 2][(i & 3) * 4 + j] += attn_taken((float)v[j]);
      }
    }
  }

  const float sum = l_run + __shfl_xor(l_run, 32), true_sum = LSE ? l_true + __shfl_xor(l_true, 32) : sum;
  if (row < w.rows) {
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum, lse2 = none ? -INFINITY : m_run * scale2 + __builtin_amdgcn_logf(true_sum);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = db * 32 + 8 * i + 4 * h;
        if (FULL || d < p.D) attn_store<bf16>(p, w, row, d, f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]}, inv, lse2);
      }
  }
}

template <int DP>
hipError_t launch_dp(const PagedAttnP& p, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const auto go = [&](auto kernel) { kernel<<<grid, kPromptWaves * 64, 4 * kTile * DP * 2, st>>>(p); };
  if (p.lse)
    go(p.D == DP ? paged_attn_prompt_kernel<DP, kPromptWaves, true, true> : paged_attn_prompt_kernel<DP, kPromptWaves, false, true>);
  else
    go(p.D == DP ? paged_attn_prompt_kernel<DP, kPromptWaves, true, false> : paged_attn_prompt_kernel<DP, kPromptWaves, false, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn_prompt(const PagedAttnP& p, hipStream_t st) {
  return p.D <= 64 ? launch_dp<64>(p, st) : launch_dp<128>(p, st);
}

}  // namespace tsd
