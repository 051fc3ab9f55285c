// tsd_paged_attn_static on bf16 caches, the join of split sequences, and the entry points.
//
// One wavefront takes 32 keys a step for 16 * MT rows:
//   S^T = K Q^T   two 16x16x32 MFMAs per 32 dims and row tile; key rows are permuted so that lane group g = lane / 16 ends up with the
//                 scores of the 8 consecutive keys 8g .. 8g + 7 for row lane % 16, which is the A operand of the next product;
//   online softmax in fp32, base 2 (running maximum and sum per row, shared by its 4 lanes).  The weights are rounded to bf16, the matrix
//                 instruction's operand, and the sum is that of the rounded ones: a weight's error of up to 2^-8 then moves the result only by
//                 the share of its value's distance from the mean;
//   O += P V      V rows are fetched with 16-byte loads, parked in LDS and picked up transposed with ds_read_b64_tr_b16.
// Few rows are memory bound: the next step's keys and values are asked for before this one's softmax, into the registers that its own
// left.  One token of 64 sequences of 100 to 8192 keys, 32 heads over 8 of 128: 212 us for 254387 keys in all, 4.9 TB/s (a copy reaches 5.2, eight other
// draws of lengths 195 to 237 us, 4.7 to 5.0); 16 heads over 4 of 256, 2000 keys each: 97 us, 5.4 TB/s; 7 tokens of 512 sequences
// of 80 keys, 16 heads of 64: 44 us, 4.1 TB/s, a wavefront's three steps behind two trips for its lengths and pages; 5 tokens of one
// sequence of 32768 keys, 32 heads over 8 of 128: 36.5 us, 3.7 TB/s, of which the join is 5 and the first and last trips some 6.  Windows read what they leave
// visible: one token of 64 sequences, of the last 4096 keys and the first four of up to 16384, 32 heads over 8 of 128, 179 us, 946 MB, 5.3 TB/s; of the last 1024
// of one sequence of 20000 10.3 us, trips.
#include <algorithm>
#include <cmath>

#include "paged_attn.h"

namespace tsd {
namespace {

constexpr int v_stride(int dp) { return dp + 16; }  // V row in LDS: 32 bytes more than its dims, so that 8 rows fall on different banks

template <int M, int DP, int MT, bool FULL>  // M: AttnMask; FULL: head_dim is DP
__global__ __launch_bounds__(kAttnWaves * 64, DP <= 128 ? 2 : 1) void paged_attn_bf16_kernel(const PagedAttnP p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KK = DP / 32, NB = DP / 16, VS = v_stride(DP), NV = DP / 16, VC = DP / 8;
  constexpr int kSure = FULL ? DP : DP == 32 ? 8 : DP == 64 ? 40 : DP == 96 ? 72 : DP == 128 ? 104 : 136;  // dims that every head of this kernel has
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
  const bf16* kbase = reinterpret_cast<const bf16*>(p.cache.k) + w.hk * p.cache.head_stride;
  const bf16* vbase = reinterpret_cast<const bf16*>(p.cache.v) + w.hk * p.cache.head_stride;
  bf16* vt = reinterpret_cast<bf16*>(smem) + wave * 32 * VS;
  const bf16x8 zero = {};

  bf16x8 qf[MT][KK];
  decltype(sight(0)) sees[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = w.row0 + mt * 16 + qi;
    sees[mt] = sight(row);
    const int r = min(row, w.rows - 1), t = r / p.G, h = w.hk * p.G + r - t * p.G;
    const bf16* q = reinterpret_cast<const bf16*>(p.q.p) + w.b * p.q.sb + t * p.q.st + h * p.q.sh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = kk * 32 + g * 8;
      qf[mt][kk] = kk * 32 + 32 <= kSure || d < p.D ? *reinterpret_cast<const bf16x8*>(q + d) : zero;
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
        const bool in = kk * 32 + 32 <= kSure || d < p.D;
        kf[bi][kk] = *reinterpret_cast<const bf16x8*>(k + (in ? d : 0));
        if (!in) kf[bi][kk] = zero;
      }
    }
  };
  auto load_v = [&](long off) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * 64 + lane, r = c / VC, d = (c - r * VC) * 8;
      vf[i] = *reinterpret_cast<const bf16x8*>(vbase + __shfl(off, r) + (FULL || d < p.D ? d : 0));  // (dims from D on: anything, never written)
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
    const bool whole = valid == 0xFFFFFFFFu && attn_all_see<M>(p, w, sb, 32);  // every row of the tile sees every key
    unsigned live[MT] = {};  // of the lane's 8 keys
    if (!whole) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if constexpr (M == kCausal)
          live[mt] = (valid & attn_bits(sees[mt].sees - sb)) >> (8 * g);
        else
          live[mt] = (valid & seen(sees[mt], sb)) >> (8 * g);
      }
      // keys that are not there hold anything; their weights are 0, and so must the values be
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (!(valid >> ((i * 64 + lane) / VC) & 1)) vf[i] = zero;
      if (attn_mixed<M>(p, w, sb, 32)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) odd |= attn_take_out(vf[i]);
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
    off = later;

    bf16x8 pf[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float s[8], e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = sc[mt][j >> 2][j & 3] * p.scale2;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!(live[mt] >> j & 1)) s[j] = -INFINITY;
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
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      typedef short short4v __attribute__((ext_vector_type(4)));
      short4v hv[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16* src = vt + (8 * g + 4 * half + (qi >> 2)) * VS + nb * 16 + 4 * (qi & 3);
        hv[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)src);
      }
      const bf16x8 vv = __builtin_bit_cast(bf16x8, __builtin_shufflevector(hv[0], hv[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) o[mt][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[mt], vv, o[mt][nb], 0, 0, 0);
    }
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
      for (int nb = 0; nb < NB; ++nb) {
        const float v = FULL || nb * 16 + qi < p.D ? attn_taken((float)vbase[at + nb * 16 + qi]) : 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (reached >> (4 * mt + r) & 1) o[mt][nb][r] += v;
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
  if (p.slots) attn_finish<bf16>(p, w, 16 * MT, reinterpret_cast<float*>(smem));
}

// Joins the chunks of a row: WPR wavefronts take one, their lanes 4 dims each, as many groups of lanes as a wavefront has room for
// every so many chunks.
template <typename T, int WPR>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(const PagedAttnP p) {
  __shared__ float part[256 * 5];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long r = blockIdx.x * (4l / WPR) + wave / WPR;
  const bool there_is = r < (long)p.B * p.T * p.Hq;
  const int h = (int)(r % p.Hq), t = (int)(r / p.Hq % p.T), b = there_is ? (int)(r / p.Hq / p.T) : 0;
  const bool live = there_is && t < attn_new(p, b);
  const int chunks = live ? attn_chunks(p, attn_len(p, b)) : 0;
  const int lpr = p.D / 4, groups = 64 / lpr, d = (lane % lpr) * 4, grp = lane / lpr;
  const long row = ((long)b * p.splits * p.T + t) * p.Hq + h, step = (long)p.T * p.Hq;  // of chunk 0, and between chunks
  float mm = -INFINITY;
  for (int s = lane; s < chunks; s += 64) mm = fmaxf(mm, p.part_lse[row + s * step]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (grp < groups) {
    constexpr int U = 4;  // chunks whose loads are in flight together
    const int every = WPR * groups;
    for (int s0 = wave % WPR * groups + grp; s0 < chunks; s0 += U * every) {
      float l[U];
      f32x4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = min(s0 + u * every, chunks - 1);
        l[u] = p.part_lse[row + s * step];
        y[u] = *reinterpret_cast<const f32x4*>(p.part_o + (row + s * step) * p.D + d);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (s0 + u * every >= chunks || l[u] == -INFINITY) continue;  // (a chunk without keys of this row)
        const float f = __builtin_amdgcn_exp2f(l[u] - mm);
        sum += f;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += f * y[u][j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[threadIdx.x * 5 + j] = o[j];
  part[threadIdx.x * 5 + 4] = sum;
  __syncthreads();
  if (!live || grp || wave % WPR) return;
  for (int v = 0; v < WPR; ++v)
    for (int i = v == 0; i < groups; ++i) {
      const float* x = part + (threadIdx.x + v * 64 + i * lpr) * 5;
      sum += x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += x[j];
    }
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
  attn_write<T>(p, b, t, h, d, o, inv, none ? -INFINITY : mm + __builtin_amdgcn_logf(sum));
}

template <typename T>
hipError_t launch_join(const PagedAttnP& p, hipStream_t st) {
  const int64_t rows = (int64_t)p.B * p.T * p.Hq;
  if (p.splits > 8)
    paged_attn_join_kernel<T, 4><<<(unsigned)rows, 256, 0, st>>>(p);
  else
    paged_attn_join_kernel<T, 1><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(p);
  return hipGetLastError();
}

template <int M, int DP>
hipError_t launch_dp(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  const dim3 grid((unsigned)((long)p.B * p.Hkv * p.row_tiles * p.splits));
  const size_t stage = (size_t)waves * 32 * v_stride(DP) * 2, join = (size_t)waves * 16 * ((DP + 4) * 4 + 8);
  const size_t lds = stage > join ? stage : join;
  const auto go = [&](auto kernel) { kernel<<<grid, waves * 64, lds, st>>>(p); };
  if (mt == 1)
    go(p.D == DP ? paged_attn_bf16_kernel<M, DP, 1, true> : paged_attn_bf16_kernel<M, DP, 1, false>);
  else if constexpr (DP <= 128)
    go(p.D == DP ? paged_attn_bf16_kernel<M, DP, 2, true> : paged_attn_bf16_kernel<M, DP, 2, false>);
  return hipGetLastError();
}

// What the sizes make of a call.
//
// Chunks: as many as give every compute unit one workgroup (256 in all: a step more and some get two, 32 x 1 x 1024 keys of 8 heads 33.7 us,
// 36 x 896 42.9), none shorter than a step of all wavefronts, and of at most 1024 keys where up to four workgroups a compute unit would
// otherwise go by the longest sequence (64 ragged sequences of up to 8192: whole 239 us, 1024 keys 217, 256 keys 256).  With more
// workgroups than that, sequences stay whole.  At most 16384 workgroups, most of them idle, where max_len says much more than lengths are.
// For many rows, whose parts are much to write and join, chunks are no shorter than an eighth of max_len in whole tiles of 64 keys, or than 256, and
// up to 256 keys stay whole (128 rows of 8 heads of 64: 11.1 us, in two 14.0).  us at 512 keys with chunks of 64, 128 and 256: 68 rows of 2 heads of
// 128 12.0, 14.7, 18.2, 300 rows of 4 of 80 14.0, 16.2, 19.8, but with 64 and 256 128 rows of 32 of 128 23.6, 20.8; at 1000 keys with 128 and 256: 128
// rows of 8 of 128 15.1, 18.1; at 2000 keys with 128 and 256: 256 rows of 8 of 128 26.2, 20.2, 68 rows of 2 14.6, 18.2.
// Kernel: the one for many rows from 65 rows a key head on (68 of 8 heads of 128, us for 64 sequences of up to 8192: 296 against 629; 120 of 4 of 80, 32
// of up to 2000: 54 against 68), and from 33 on where heads are wide and workgroups enough (40 of 8 of 128, 64 sequences: 276 against 441, 8: 49
// against 66; but 36 of 4 of 64, 128 sequences of up to 2000: 62 and 62).  Heads above 128 have none: 2 x 1024 tokens behind 2048, 16 heads over 4 of
// 256, take 423 us (0.20 PFLOP/s) in tiles of 16 rows.
// Joins: by the last workgroup where that is little work for one (12 chunks of 9 rows of 80: 17.5 us against 19.0 with a second launch, 8 of 8 rows of
// 64 9.0 and 10.6; 32 of 20 rows of 128 47.5 and 39.3), and not for many rows (2 chunks of 128 rows of 64 24.5 and 15.4).
// Wavefronts: four share a workgroup's keys, or, where there are workgroups enough and a few steps in all, one takes them (512 x 16 of 80 keys
// 45.9 us, two 46.8, four 52.0).
// The rules above were swept with causal calls, and windows and trees take them over; `least` holds a single sequence's tree at 256 keys a chunk, as it does
// a causal call (26 nodes behind 1974 keys: 64 workgroups).
// All of this goes by the places that a row tile may have, where windows leave fewer of them than max_len.  Windows make lengths alike, and a tree's rows are
// many to join: their chunks are longer.  Few rows (us with 1024, some 3000 keys and whole): 64 tokens at a window of 4096, 32 heads over 8 of 128, 191, 190, 179,
// 32 100, 96, 90, but 16 (2048) 53, 52, 66; trees of 8 nodes over up to 16384 keys, 16 sequences 154, 146 (2560: 140), 143 (8192), up to 3000 keys, 64 sequences 136, 121, 121; of
// 64, 16 heads of 64, 296, 261, 246 (4096).  Their border, 4608 places, lies between two sides that are close, but for few sequences: one token at a window, 32 heads
// over 8 of 128, us in chunks of 1024, 2560, 4096 and whole, for 16, 32, 64 and 100 sequences: window 3000 40, 37, 37, 37; 87, 80, 80, 80; 154, 145, 146, 145; 243, 257,
// 256, 256; 4096 50, 51, 54, 54; 116, 115, 108, 109; 207, 202, 197, 197; 326, 325, 346, 346; 5000 70, 64, 86, 87; 140, 137, 131, 131; 251, 246, 240, 240; 393, 400, 421,
// 421; 8192 114, 122, 111, 144; 222, 219, 217, 211; 407, 398, 393, 387; 638, 623, 648, 686; 16384 221, 221, 213, 279; 440, 429, 426, 416; 799, 791, 779, 768; 1251,
// 1230, 1238, 1367.  (Whole is best, by up to 7 %, where workgroups are a multiple of the compute units, at any window, and parts where they are not: the border
// gives some of the one away above it, up to 5 %, and of the other below, up to 7 %.)  Trees of many rows: chunks for some 512 workgroups, of at most 2560 keys, as
// long as the tiles alone do not fill the card: 64 nodes over up to 16384 keys, 32 heads over 8 of 128, us with 512, 1024, 2048, 2752, 4096, 8192: 16 sequences 352, 307, 263,
// 261, 297, 319; 4 sequences 109, 99, 92, 109, 135, 242; 2 sequences 62, 59, 75, 94, 132, 236; 1 sequence (256: 39) 41, 46, 72; 8 sequences of 16000 307, 258, 220,
// 223, 210, 258; 32 sequences of up to 8000 410, 289, 275, 272, 299, 307; but 16 of up to 2000 79, 74, whole 68, 64 of up to 4096 444, 407, 386, whole 305.
// Parts of windows and trees take 256 MiB at most: by keys alone, 16 trees of 64 nodes over up to 131072 had 806 MiB, 64 over up to 65536 838, and were no faster
// (chunks of 2624 keys and of 8768: 2060 and 1995 us; of 5056 and 21888: 4016 and 3981; 4 of 256 nodes over up to 65536, of 2560 and 4416: 1071 and 1017).
// In fp32, where products bound, and of lengths that windows make alike, tiles of 16 rows fill the card better up to 128 rows: 51 rows at a window of 500, 24
// sequences, 4 heads of 80 34 us against 37, of 128 32 and 43, 200 sequences 118 and 168, but 256 rows, 16 sequences, 8 heads of 128, 307 and 247.  Trees over whole
// caches have the same rule, and it fits those of one sequence and short ones (us in tiles of 16 and 32 rows; 51 rows of 4 heads of 80: 1 sequence of 12000 keys 31, 34, 8
// of up to 3000 46, 47, 24 of up to 500 30, 37), not many long ones, whose keys the tiles fetch anew (24 of up to 3000 132, 106; 27 rows of 4 heads of 128, 64 sequences, up
// to 500 48, 38, 3000 237, 158, 12000 905, 583; of 64 96, 97 at 3000, 424, 314 at 12000; 128 rows of 8 of 128, 4 sequences, 12000 365, 345).
struct AttnPlan {
  bool prompt;  // the kernel for many rows
  int mt, waves, row_tiles, splits, chunk, reach;
  bool joins;   // the last workgroup of a tile joins its chunks
};

// What a call says of its mask.
struct AttnAsk {
  AttnMask mask;
  int window, sinks;
  const int32_t* parents;
  int parents_stride;
};
constexpr int kMostTokens = 1 << 30;
constexpr int64_t kMostParts = 256 << 20;  // bytes of a call's parts, but for causal calls
constexpr AttnAsk kAllKeys = {kCausal, kMostTokens, 0, nullptr, 0};

AttnPlan attn_plan(const AttnAsk& ask, int dtype, int B, int T, int Hq, int Hkv, int D, int max_len) {
  AttnPlan a;
  const int64_t rows = (int64_t)T * (Hq / Hkv);
  a.prompt = dtype == TSD_BF16 && D <= 128 && (rows > 64 || (rows > 32 && D > 96 && (int64_t)B * Hkv >= 64));
  const bool small = ask.mask != kCausal && dtype == TSD_F32 && rows <= 128;
  a.mt = rows <= 16 || D > 128 || small ? 1 : 2;
  const int tile_rows = a.prompt ? kPromptRows : 16 * a.mt;
  a.row_tiles = (int)((rows + tile_rows - 1) / tile_rows);
  // (the tokens that a tile's rows may belong to; a tree's nodes are at most as far apart as there are nodes)
  const int64_t tokens = ask.mask == kTree ? T : std::min<int64_t>(T, (tile_rows + Hq / Hkv - 2) / (Hq / Hkv) + 1);
  a.reach = (int)std::min<int64_t>(kMostTokens, (int64_t)ask.sinks + ask.window + tokens - 1);
  max_len = std::min(max_len, a.reach);
  const int64_t base = (int64_t)B * Hkv * a.row_tiles, steps = (max_len + 31) / 32;  // workgroups where nothing is split
  a.waves = a.prompt ? kPromptWaves : (int)std::min<int64_t>(base >= 1024 && steps <= 4 ? 1 : D > 128 ? 2 : kAttnWaves, steps);
  const int64_t step = a.prompt ? 64 : 32 * a.waves;
  int64_t chunk = max_len;
  const bool tall = a.prompt && a.row_tiles > 1;  // (sums of many rows cost more to join than unequal lengths do)
  if (base < (tall ? 256 : 1024)) {
    const int64_t most = tall ? max_len : ask.mask == kCausal ? 1024 : max_len <= 4608 ? max_len : 2560;
    chunk = std::min<int64_t>(max_len * base / 256, most);
    chunk = chunk < step + step / 4 ? step : (chunk + step - 1) / step * step;
  }
  // (many rows: not less than is worth joining)
  const int64_t least = !a.prompt ? 1 : max_len <= 256 ? 256 : std::min<int64_t>(256, (max_len + 511) / 512 * 64);
  if (a.prompt && ask.mask == kTree) {
    chunk = std::max<int64_t>(max_len * base / (base < 32 ? 1024 : 512), base >= 256 ? 2048 : std::min(8 * base, (int64_t)max_len / 4));
    chunk = std::max(least, std::min(chunk, 2560 * std::max<int64_t>(1, base / 512)));
    const int64_t parts = std::max<int64_t>(1, (max_len + chunk / 2) / chunk);  // (alike)
    chunk = (max_len + parts - 1) / parts;
  }
  chunk = std::max(chunk, least);
  if (ask.mask != kCausal) {
    const int64_t parts = std::max<int64_t>(1, kMostParts / ((int64_t)B * T * Hq * (D + 1) * 4));
    chunk = std::max(chunk, (max_len + parts - 1) / parts);
  }
  if (ask.mask != kCausal && max_len - chunk < chunk / 4) chunk = max_len;
  chunk = std::min<int64_t>(std::max(chunk, max_len * base / 16384), max_len);  // (a sequence that stays whole: no longer than it is)
  chunk = (chunk + step - 1) / step * step;
  a.chunk = (int)chunk;
  a.splits = (int)((max_len + chunk - 1) / chunk);
  a.joins = !a.prompt && a.splits > 1 && a.splits <= 16 && base < 256 && a.splits * std::min<int64_t>(rows, tile_rows) * D <= 16384;
  return a;
}

int check_attn(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len) {
  if (B < 1 || T < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1 and T >= 1");
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % cache->n_kv_heads)
    return fail_no_handle(TSD_E_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 1024");
  if (max_len < 1 || max_len > kMostTokens) return fail_no_handle(TSD_E_INVALID_ARG, "max_len must be 1..2^30");
  if ((int64_t)B * T * n_q_heads > INT32_MAX) return fail_no_handle(TSD_E_OUT_OF_RANGE, "B * T * n_q_heads beyond 2^31 - 1");
  return TSD_OK;
}

// The workspace: sums, logarithms, slots.
size_t attn_part_bytes(const AttnPlan& a, int B, int T, int Hq, int D) { return ((size_t)B * a.splits * T * Hq * (D + 1) * 4 + 7) / 8 * 8; }
size_t attn_bytes(const AttnPlan& a, int B, int T, int Hq, int Hkv, int D) {
  if (a.splits == 1) return 0;
  return (attn_part_bytes(a, B, T, Hq, D) + (size_t)B * Hkv * a.row_tiles * a.splits * 8 + 255) / 256 * 256;
}

template <int M>
hipError_t launch_mask(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  if (p.D <= 32) return launch_dp<M, 32>(p, mt, waves, st);
  if (p.D <= 64) return launch_dp<M, 64>(p, mt, waves, st);
  if (p.D <= 96) return launch_dp<M, 96>(p, mt, waves, st);
  if (p.D <= 128) return launch_dp<M, 128>(p, mt, waves, st);
  return launch_dp<M, 256>(p, mt, waves, st);
}

}  // namespace

hipError_t launch_paged_attn_bf16(const PagedAttnP& p, int mt, int waves, hipStream_t st) {
  return p.mask == kCausal ? launch_mask<kCausal>(p, mt, waves, st) : p.mask == kWindow ? launch_mask<kWindow>(p, mt, waves, st) : launch_mask<kTree>(p, mt, waves, st);
}

}  // namespace tsd

using namespace tsd;

namespace {

// A window of 0: every key before a row's own.
int check_ask(const AttnAsk& ask, int32_t T) {
  if (ask.mask == kCausal) return TSD_OK;
  if (ask.window < 1) return fail_no_handle(TSD_E_INVALID_ARG, ask.mask == kTree ? "window must not be negative" : "window must be at least 1");
  if (ask.sinks < 0) return fail_no_handle(TSD_E_INVALID_ARG, "sinks must not be negative");
  if (ask.mask == kTree && T > kTreeNodes) return fail_no_handle(TSD_E_OUT_OF_RANGE, "a tree has at most 256 nodes");
  return TSD_OK;
}

int attn_workspace(const AttnAsk& ask, const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len, size_t* bytes_host) {
  int rc = check_attn(cache, B, T, n_q_heads, max_len);
  if (rc || (rc = check_ask(ask, T))) return rc;
  if (!bytes_host) return fail_no_handle(TSD_E_INVALID_ARG, "bytes_host must not be NULL");
  const AttnPlan a = attn_plan(ask, cache->dtype, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim, max_len);
  *bytes_host = attn_bytes(a, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim);
  return TSD_OK;
}

int attn_call(const AttnAsk& ask, const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* out,
              float* lse_dev, const int32_t* lens_dev, const int32_t* n_new_dev, int32_t max_len, float scale, void* workspace_dev,
              size_t workspace_bytes, void* stream) {
  int rc = check_attn(cache, B, T, n_q_heads, max_len);
  if (rc || (rc = check_ask(ask, T))) return rc;
  const int es = type_bytes(cache->dtype);
  if ((rc = check_rows(q, es, "q")) || (rc = check_rows(out, es, "out"))) return rc;
  if (!lens_dev) return fail_no_handle(TSD_E_INVALID_ARG, "lens_dev must not be NULL");
  if (ask.mask == kTree && !ask.parents) return fail_no_handle(TSD_E_INVALID_ARG, "parents_dev must not be NULL");
  if (ask.mask == kTree && ask.parents_stride && ask.parents_stride < T) return fail_no_handle(TSD_E_INVALID_ARG, "parents_stride must be 0 or at least T");
  if (!std::isfinite(scale)) return fail_no_handle(TSD_E_INVALID_ARG, "scale must be finite");
  const AttnPlan a = attn_plan(ask, cache->dtype, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim, max_len);
  const size_t need = attn_bytes(a, B, T, n_q_heads, cache->n_kv_heads, cache->head_dim);
  if (need && (!workspace_dev || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)))
    return fail_no_handle(TSD_E_INVALID_ARG, "workspace: needs the bytes that the call for its size gives for these sizes, 16-byte aligned");
  if ((int64_t)B * cache->n_kv_heads * a.row_tiles * a.splits > max_workgroups(64 * kAttnWaves) ||
      (a.splits > 1 && (int64_t)B * T * n_q_heads > max_workgroups(256)))
    return fail_no_handle(TSD_E_OUT_OF_RANGE, "more than 2^24 - 1 workgroups");
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
  p.slots = a.joins ? reinterpret_cast<uint64_t*>(static_cast<char*>(workspace_dev) + attn_part_bytes(a, B, T, n_q_heads, cache->head_dim)) : nullptr;
  p.tag = a.joins ? new_tag() : 0;
  p.mask = ask.mask;
  p.window = ask.window;
  p.sinks = ask.sinks;
  p.reach = a.reach;
  p.parents = ask.parents;
  p.parents_stride = ask.parents_stride;
  const hipStream_t st = (hipStream_t)stream;
  hipError_t e = a.prompt                   ? launch_paged_attn_prompt(p, st)
                 : cache->dtype == TSD_BF16 ? launch_paged_attn_bf16(p, a.mt, a.waves, st)
                                            : launch_paged_attn_f32(p, a.mt, a.waves, st);
  if (e == hipSuccess && a.splits > 1 && !a.joins) e = cache->dtype == TSD_BF16 ? launch_join<bf16>(p, st) : launch_join<float>(p, st);
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("paged attention launch: ") + hipGetErrorString(e));
}

AttnAsk window_ask(int32_t window, int32_t sinks) { return {kWindow, std::min<int>(window, kMostTokens), std::min<int>(sinks, kMostTokens), nullptr, 0}; }
AttnAsk tree_ask(int32_t window, int32_t sinks, const int32_t* parents, int32_t stride) {
  return {kTree, window ? std::min<int>(window, kMostTokens) : kMostTokens, std::min<int>(sinks, kMostTokens), parents, stride};
}

}  // namespace

extern "C" int tsd_paged_attn_workspace(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len, size_t* bytes_host) {
  return attn_workspace(kAllKeys, cache, B, T, n_q_heads, max_len, bytes_host);
}

extern "C" int tsd_paged_attn_static(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* out,
                                     float* lse_dev, const int32_t* lens_dev, const int32_t* n_new_dev, int32_t max_len, float scale,
                                     void* workspace_dev, size_t workspace_bytes, void* stream) {
  return attn_call(kAllKeys, cache, B, T, n_q_heads, q, out, lse_dev, lens_dev, n_new_dev, max_len, scale, workspace_dev, workspace_bytes, stream);
}

extern "C" int tsd_window_attn_workspace(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len, int32_t window,
                                         int32_t sinks, size_t* bytes_host) {
  return attn_workspace(window_ask(window, sinks), cache, B, T, n_q_heads, max_len, bytes_host);
}

extern "C" int tsd_window_attn_static(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* out,
                                      float* lse_dev, const int32_t* lens_dev, const int32_t* n_new_dev, int32_t max_len, int32_t window,
                                      int32_t sinks, float scale, void* workspace_dev, size_t workspace_bytes, void* stream) {
  return attn_call(window_ask(window, sinks), cache, B, T, n_q_heads, q, out, lse_dev, lens_dev, n_new_dev, max_len, scale, workspace_dev,
                   workspace_bytes, stream);
}

extern "C" int tsd_tree_attn_workspace(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, int32_t max_len, int32_t window,
                                       int32_t sinks, size_t* bytes_host) {
  return attn_workspace(tree_ask(window, sinks, nullptr, 0), cache, B, T, n_q_heads, max_len, bytes_host);
}

extern "C" int tsd_tree_attn_static(const tsd_paged_cache* cache, int32_t B, int32_t T, int32_t n_q_heads, const tsd_rows* q, const tsd_rows* out,
                                    float* lse_dev, const int32_t* lens_dev, const int32_t* n_new_dev, const int32_t* parents_dev,
                                    int32_t parents_stride, int32_t max_len, int32_t window, int32_t sinks, float scale, void* workspace_dev,
                                    size_t workspace_bytes, void* stream) {
  return attn_call(tree_ask(window, sinks, parents_dev, parents_stride), cache, B, T, n_q_heads, q, out, lse_dev, lens_dev, n_new_dev, max_len,
                   scale, workspace_dev, workspace_bytes, stream);
}
