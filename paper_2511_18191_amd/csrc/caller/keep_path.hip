// tsd_keep_path_static: the kept nodes of a tree, wherever their slots lie, move together behind the tokens that the cache held.
//
// Slot held + path[i] goes to slot held + i.  A path goes up (parents come before their children), so that path[i] >= i: what is read for i lies at or
// behind what is written for i, and only writes for later i reach it.  A lane takes one 16-byte column of the keys' or values' rows of a
// (layer, sequence) for the whole path, reads before it writes, and nobody else touches its column: no order between lanes matters.  (Where keys and values
// are the same rows of one pool, they are moved once: two lanes would share a column.)
//
// Every byte is read and written once: memory bound, and for few tokens the trips to the path, the table and the rows.  Eight heads of 128, bf16: 4 rows of one
// layer 3.0 us (a call 4.7), up to 8 rows of 64 sequences and 24 layers, 44 MB moved, 11.3 us (3.9 TB/s; a copy reaches 5.0 and would need 8.8).
#include "paged_cache.h"

namespace tsd {
namespace {

struct KeepP {
  PagedView cache;  // strides and pools in bytes here
  long layer_stride;
  const int* held;
  const int* path;  // [B][N]
  int B, N, cols, per_head;  // 16-byte columns of a row of keys, and of one head
  int all;                   // columns of keys and values
};

__global__ __launch_bounds__(256) void keep_path_kernel(const KeepP p) {
  typedef unsigned Words __attribute__((ext_vector_type(4)));
  const int parts = (p.all + 255) / 256;
  unsigned i = blockIdx.x;
  const int part = i % parts;
  i /= parts;
  const int b = i % p.B, layer = i / p.B;
  const int col = part * 256 + threadIdx.x, lane = threadIdx.x & 63;
  const int* path = p.path + (long)b * p.N;
  const int* table = p.cache.table + (long)b * p.cache.table_stride;
  const int held = p.held[b];
  const bool values = col >= p.cols;
  const int c = values ? col - p.cols : col, head = c / p.per_head;
  char* pool = (values ? p.cache.v : p.cache.k) + layer * p.layer_stride + head * p.cache.head_stride + (c - head * p.per_head) * 16;
  const bool live = col < p.all;
  int before = -1;
  for (int base = 0; base < p.N; base += 64) {
    // 64 entries of the path at a time, as far as it goes up
    const int at = base + lane < p.N ? path[base + lane] : -1;
    int prev = __shfl_up(at, 1);
    if (lane == 0) prev = before;
    const unsigned long long up = __ballot(at > prev && at < p.N);
    const int n = __builtin_ctzll(~up | (1ull << 63)) + (up == ~0ull);  // (how many lanes from the first on)
    long from = -1, to = -1;
    if (lane < n && at != base + lane && held >= 0 && held <= (1 << 30)) {
      const int x = held + at, y = held + base + lane;
      from = paged_row(p.cache, paged_entry(p.cache, table, x), x);
      to = paged_row(p.cache, paged_entry(p.cache, table, y), y);
    }
    const unsigned long long moves = __ballot(from >= 0 && to >= 0);
    constexpr int U = 8;  // rows on their way together
    for (int k0 = 0; k0 < n; k0 += U) {
      if (!(moves >> k0 & 0xFF)) continue;
      Words x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long off = __shfl(from, k0 + u);
        if (live && (moves >> (k0 + u) & 1)) x[u] = *reinterpret_cast<const Words*>(pool + off);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long off = __shfl(to, k0 + u);
        if (live && (moves >> (k0 + u) & 1)) *reinterpret_cast<Words*>(pool + off) = x[u];
      }
    }
    if (n < 64) return;
    before = __shfl(at, 63);
  }
}

}  // namespace
}  // namespace tsd

using namespace tsd;

extern "C" int tsd_keep_path_static(const tsd_paged_cache* cache, int32_t n_layers, int64_t layer_stride, int32_t B, int32_t N, const int32_t* held_dev,
                                    const int32_t* path_dev, void* stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (B < 1 || N < 1 || n_layers < 1) return fail_no_handle(TSD_E_INVALID_ARG, "need B >= 1, N >= 1 and n_layers >= 1");
  if (N > kTreeNodes) return fail_no_handle(TSD_E_OUT_OF_RANGE, "a tree has at most 256 nodes");
  if (!held_dev || !path_dev) return fail_no_handle(TSD_E_INVALID_ARG, "held_dev and path_dev must not be NULL");
  const int es = type_bytes(cache->dtype);
  if (layer_stride < 0 || (layer_stride * es & 15)) return fail_no_handle(TSD_E_INVALID_ARG, "layer_stride must be a multiple of 16 bytes, not negative");
  if (n_layers > 1 && !layer_stride) return fail_no_handle(TSD_E_INVALID_ARG, "layer_stride must not be 0 beside several layers: each would move the same rows");
  KeepP p;
  p.cache = cache_view(*cache);
  p.cache.page_stride *= es;
  p.cache.token_stride *= es;
  p.cache.head_stride *= es;
  p.layer_stride = layer_stride * es;
  p.held = held_dev;
  p.path = path_dev;
  p.B = B;
  p.N = N;
  p.per_head = cache->head_dim * es / 16;
  p.cols = cache->n_kv_heads * p.per_head;
  p.all = cache->k_dev == cache->v_dev ? p.cols : 2 * p.cols;
  const int64_t parts = (p.all + 255) / 256;
  if ((int64_t)B * n_layers > max_workgroups(256) / parts) return fail_no_handle(TSD_E_OUT_OF_RANGE, "more than 2^24 - 1 workgroups");
  keep_path_kernel<<<(unsigned)(parts * B * n_layers), 256, 0, (hipStream_t)stream>>>(p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSD_OK : fail_no_handle(TSD_E_HIP, std::string("kept path launch: ") + hipGetErrorString(e));
}
