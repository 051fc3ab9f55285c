// Attention of new tokens over a caller's paged cache: what its kernels share (paged_attn.hip on bf16 caches,
// paged_attn_prompt.hip on bf16 caches where rows are many, paged_attn_f32.hip on fp32 ones).
//
// Rows: the T new tokens and the G = Hq / Hkv query heads of one key head are rows t * G + g of one product, in tiles, so that a
// key head's keys and values are read once for all of them.  Row of token t sees keys j < len - n_new + t + 1.
//
// Split: the keys of a sequence go in chunks of `chunk`; a workgroup takes one (sequence, key head, row tile, chunk), its wavefronts take
// its steps of 32 keys in turn, each with a running maximum and sum of its own, joined in LDS at the end.  Where a sequence may
// have several chunks, each leaves its rows' normalised sums and their logarithm (base 2) in the workspace.  They are joined by the workgroup
// of a (sequence, key head, row tile) that comes last (last_arriver.h), or, where that is much for one workgroup or rows are many, by a second launch.
#pragma once
#include "last_arriver.h"
#include "paged_cache.h"

namespace tsd {

struct PagedAttnP {
  PagedView cache;
  RowsView q, out;
  float* lse;        // [B][T][Hq] natural logarithms (NULL: none)
  const int* lens;
  const int* n_new;  // NULL: T
  int B, T, Hq, Hkv, G, D;
  int row_tiles, splits, chunk;
  float scale2;      // scale * log2(e)
  float* part_o;     // [B][splits][T][Hq][D] (splits > 1)
  float* part_lse;   // [B][splits][T][Hq]
  uint64_t* slots;   // [B][Hkv][row_tiles][splits], or NULL: a second launch joins
  uint64_t tag;
};

constexpr int kAttnWaves = 4;  // most wavefronts a workgroup has

// launches of one type's kernels: mt row tiles of 16 a workgroup, `waves` wavefronts
hipError_t launch_paged_attn_bf16(const PagedAttnP& p, int mt, int waves, hipStream_t st);
constexpr int kPromptWaves = 4, kPromptRows = 128;
hipError_t launch_paged_attn_prompt(const PagedAttnP& p, hipStream_t st);  // bf16, head_dim <= 128: row tiles of kPromptRows
hipError_t launch_paged_attn_f32(const PagedAttnP& p, int mt, int waves, hipStream_t st);

#if defined(__HIPCC__)
// What a workgroup works on.
struct AttnWork {
  int b, hk, tile, split;
  int len, n_new;     // of the sequence
  int rows;           // live rows of the key head: n_new * G
  int row0;           // the tile's first row
  int see_first, see_last;  // keys that the tile's first and last rows see
  int key0, key1;     // this workgroup's keys
  bool split_out;     // its rows' sums go to the workspace
  bool idle;          // no rows or no chunk: nothing to write
};

// Chunks of a sequence that hold keys (at least one, which then writes the empty rows).
__device__ __forceinline__ int attn_chunks(const PagedAttnP& p, int len) {
  return min(p.splits, max(1, (len + p.chunk - 1) / p.chunk));
}

__device__ __forceinline__ int attn_len(const PagedAttnP& p, int b) { return min(max(p.lens[b], 0), 1 << 30); }
__device__ __forceinline__ int attn_new(const PagedAttnP& p, int b) { return p.n_new ? min(max(p.n_new[b], 0), p.T) : p.T; }

// In two halves: where, which needs no memory, and how much, which needs the lengths.  (A cache's table entries are asked for between the two.)
__device__ __forceinline__ AttnWork attn_place(const PagedAttnP& p, int tile_rows) {
  AttnWork w;
  // Key heads vary fastest: workgroups go round the XCDs, so that the row tiles of a (sequence, key head) share an XCD's L2 where
  // B * Hkv is a multiple of 8.  The last row tiles, which see the most keys, start first.
  unsigned i = blockIdx.x;
  const unsigned pairs = p.B * p.Hkv;
  const unsigned pair = i % pairs;
  i /= pairs;
  w.split = i % p.splits;
  w.tile = p.row_tiles - 1 - i / p.splits;
  w.b = pair / p.Hkv;
  w.hk = pair - w.b * p.Hkv;
  // Workgroups 256 apart tend to share a compute unit: they take different sequences, whose lengths differ.
  w.b = (w.b + i / p.splits / max(1u, 256 / pairs)) % p.B;
  w.row0 = w.tile * tile_rows;
  w.key0 = w.split * p.chunk;
  w.split_out = p.splits > 1;
  return w;
}
__device__ __forceinline__ void attn_lengths(const PagedAttnP& p, AttnWork& w, int tile_rows) {
  w.len = attn_len(p, w.b);
  w.n_new = attn_new(p, w.b);
  w.rows = w.n_new * p.G;
  const int chunks = attn_chunks(p, w.len);
  w.idle = w.row0 >= w.rows || w.split >= chunks;
  w.see_first = w.len - w.n_new + w.row0 / p.G + 1;
  w.see_last = w.len - w.n_new + (min(w.rows, w.row0 + tile_rows) - 1) / p.G + 1;
  const int end = min(w.see_last, p.cache.cols << p.cache.pt_shift);
  // (the last chunk of the grid takes what is left, so that a length beyond max_len is slow and not wrong)
  w.key1 = w.split == chunks - 1 ? end : min(end, w.key0 + p.chunk);
}

// Keys that row `row` sees (none for rows that are not there).
__device__ __forceinline__ int attn_sees(const PagedAttnP& p, const AttnWork& w, int row) {
  return row < w.rows ? w.len - w.n_new + row / p.G + 1 : 0;
}

// Offset of the cache row of key `key`, whose table entry is given, or -1 (see paged_row).
__device__ __forceinline__ long attn_key_row(const PagedAttnP& p, const AttnWork& w, int entry, int key) {
  return key < w.key1 ? paged_row(p.cache, entry, key) : -1;
}

// One step of the running softmax of a row: its lanes (q, q + 16, q + 32, q + 48) hold 8 scores each, in base 2 and -inf where the row does not
// see the key.  Returns the factor of what was summed before; e: the weights.
__device__ __forceinline__ float attn_running_max(const float (&s)[8], float& m_run, float (&e)[8]) {
  float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float m_new = fmaxf(m_run, mx);
  const float m_use = m_new == -INFINITY ? 0.f : m_new;  // (no key seen so far: every weight is 0)
  const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(s[j] - m_use);
  m_run = m_new;
  return alpha;
}

// A value that is not finite, at a key that only some rows of a tile see, must not reach the others through 0 * inf in the product of weights and values.
// Steps that hold such keys ("mixed": they end behind see_first, and rows differ) take those values out, as if they were 0; behind the last
// step they are added as they are to the rows that see them: whatever the weight, the sum is then as little finite.
// attn_take_out returns whether there were any.
__device__ __forceinline__ bool attn_take_out(bf16x8& v) {
  typedef unsigned uint4v __attribute__((ext_vector_type(4)));
  uint4v x = __builtin_bit_cast(uint4v, v);
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool lo = (x[j] & 0x7F80u) == 0x7F80u, hi = (x[j] & 0x7F800000u) == 0x7F800000u;
    x[j] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
    odd |= lo | hi;
  }
  v = __builtin_bit_cast(bf16x8, x);
  return odd;
}
__device__ __forceinline__ bool attn_take_out(f32x4& v) {
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool no = (__float_as_uint(v[j]) & 0x7F800000u) == 0x7F800000u;
    if (no) v[j] = 0.f;
    odd |= no;
  }
  return odd;
}
// What of `v` was taken out.
__device__ __forceinline__ float attn_taken(float v) { return (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? v : 0.f; }

// The first key of the mixed steps of `step` keys.
__device__ __forceinline__ int attn_mixed_from(const AttnWork& w, int step) { return w.key0 + max(w.see_first - w.key0, 0) / step * step; }

// Writes dims d .. d + 3 of a row of the output.
template <typename T>
__device__ __forceinline__ void attn_write(const PagedAttnP& p, int b, int t, int h, int d, f32x4 o, float inv, float lse2) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = (T)(o[j] * inv);
  *reinterpret_cast<T4*>(reinterpret_cast<T*>(p.out.p) + b * p.out.sb + t * p.out.st + h * p.out.sh + d) = y;
  if (d == 0 && p.lse) p.lse[((long)b * p.T + t) * p.Hq + h] = lse2 * 0.69314718055994531f;
}

// Writes dims d .. d + 3 of a row's sums, times inv: to the output, or to the workspace where a sequence may have several chunks.
template <typename T>
__device__ __forceinline__ void attn_store(const PagedAttnP& p, const AttnWork& w, int row, int d, f32x4 o, float inv, float lse2) {
  const int t = row / p.G, h = w.hk * p.G + row - t * p.G;
  if (w.split_out) {
    const long r = (((long)w.b * p.splits + w.split) * p.T + t) * p.Hq + h;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] *= inv;
    f32x4* to = reinterpret_cast<f32x4*>(p.part_o + r * p.D + d);
    if (p.slots) {
      leave(reinterpret_cast<float2*>(to), make_float2(o[0], o[1]));
      leave(reinterpret_cast<float2*>(to) + 1, make_float2(o[2], o[3]));
      if (d == 0) leave(p.part_lse + r, lse2);
    } else {
      *to = o;
      if (d == 0) p.part_lse[r] = lse2;
    }
  } else {
    attn_write<T>(p, w.b, t, h, d, o, inv, lse2);
  }
}

// Sums of a row's chunks, as they come: o and sum relative to 2^m.
struct AttnJoin {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f, m = -INFINITY;
  __device__ __forceinline__ void add(float lse2, f32x4 y) {
    if (lse2 == -INFINITY) return;  // (a chunk without keys of this row)
    const float top = fmaxf(m, lse2), a = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(lse2 - top);
    sum = sum * a + f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * a + f * y[j];
    m = top;
  }
};

// The end of a workgroup of a split call: if it came last of its (sequence, key head, row tile), it joins the chunks.  A lane takes 4 dims of a
// row; where that leaves lanes idle, groups of lanes take every so many chunks.  buf: float [blockDim.x][6] in LDS.
template <typename T>
__device__ __forceinline__ void attn_finish(const PagedAttnP& p, const AttnWork& w, int tile_rows, float* buf) {
  const int chunks = attn_chunks(p, w.len);
  uint64_t* slots = p.slots + (((long)w.b * p.Hkv + w.hk) * p.row_tiles + w.tile) * p.splits;
  if (!came_last(slots, chunks, w.split, p.tag)) return;
  const int lpr = p.D / 4, items = min(w.rows - w.row0, tile_rows) * lpr;
  const int groups = max(1, min((int)blockDim.x / items, chunks)), grp = groups > 1 ? threadIdx.x / items : 0;
  const long step = (long)p.T * p.Hq;
  for (int i = groups > 1 ? threadIdx.x - grp * items : threadIdx.x; i < items; i += blockDim.x) {
    const int lr = i / lpr, d = (i - lr * lpr) * 4, row = w.row0 + lr, t = row / p.G, h = w.hk * p.G + row - t * p.G;
    const long r = ((long)w.b * p.splits * p.T + t) * p.Hq + h;
    AttnJoin join;
    constexpr int U = 8;  // chunks whose loads are on their way together
    if (grp < groups)
      for (int s0 = grp; s0 < chunks; s0 += U * groups) {
        float l[U];
        float2 y[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long at = r + min(s0 + u * groups, chunks - 1) * step;
          l[u] = left(p.part_lse + at);
#pragma unroll
          for (int j = 0; j < 2; ++j) y[u][j] = left(reinterpret_cast<const float2*>(p.part_o + at * p.D + d) + j);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (s0 + u * groups < chunks) join.add(l[u], f32x4{y[u][0].x, y[u][0].y, y[u][1].x, y[u][1].y});
      }
    if (groups > 1) {  // (then every lane is here once)
      float* own = buf + threadIdx.x * 6;
#pragma unroll
      for (int j = 0; j < 4; ++j) own[j] = join.sum == 0.f ? 0.f : join.o[j] / join.sum;
      own[4] = join.sum == 0.f ? -INFINITY : join.m + __builtin_amdgcn_logf(join.sum);
      __syncthreads();
      if (grp) break;
      for (int v = 1; v < groups; ++v) {
        const float* x = buf + (threadIdx.x + v * items) * 6;
        join.add(x[4], f32x4{x[0], x[1], x[2], x[3]});
      }
    }
    const bool none = join.sum == 0.f;
    attn_write<T>(p, w.b, t, h, d, join.o, none ? 0.f : 1.f / join.sum, none ? -INFINITY : join.m + __builtin_amdgcn_logf(join.sum));
  }
  clear_slots(slots, chunks);
}

// Joins the wavefronts' sums of one tile of 16 rows through LDS and writes them.  O: this wavefront's sums of row `lr`, written by put(row, buf_row);
// m, l: its running maximum and sum of the lane's row (lanes of one row agree).
// buf: float [waves][16][DP + 4], ml: float2 [waves][16].
template <typename T, int DP, typename Put>
__device__ __forceinline__ void attn_join_tile(const PagedAttnP& p, const AttnWork& w, int row0, float m, float l, float* buf, float2* ml, Put put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  constexpr int RS = DP + 4;
  __syncthreads();
  put(buf + (long)wave * 16 * RS, RS);
  if (lane < 16) ml[wave * 16 + lane] = make_float2(m, l);
  __syncthreads();
  // a lane takes 4 dims of a row
  constexpr int LPR = DP / 4;
  for (int i = threadIdx.x; i < 16 * LPR; i += blockDim.x) {
    const int lr = i / LPR, d = (i - lr * LPR) * 4, row = row0 + lr;
    if (row >= w.rows || d >= p.D) continue;
    float mm = -INFINITY;
    for (int v = 0; v < waves; ++v) mm = fmaxf(mm, ml[v * 16 + lr].x);
    float sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int v = 0; v < waves; ++v) {
      const float2 x = ml[v * 16 + lr];
      if (x.y == 0.f) continue;  // saw no key of this row
      const float f = __builtin_amdgcn_exp2f(x.x - mm);
      sum += f * x.y;
      const f32x4 y = *reinterpret_cast<const f32x4*>(buf + ((long)v * 16 + lr) * RS + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * y[j];
    }
    const bool none = sum == 0.f;  // an empty row: zeros, and the logarithm of zero
    const float inv = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : mm + __builtin_amdgcn_logf(sum);
    attn_store<T>(p, w, row, d, o, inv, lse2);
  }
}
#endif

}  // namespace tsd
