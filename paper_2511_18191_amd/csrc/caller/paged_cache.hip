// Host side of the calls on a caller's paged cache: their common checks, and the rotary frequencies.
#include <cmath>

#include "paged_cache.h"

namespace tsd {

int check_cache(const tsd_paged_cache* c) {
  if (!c) return fail_no_handle(TSD_E_INVALID_ARG, "cache must not be NULL");
  if (!c->k_dev || !c->v_dev || !c->page_table_dev) return fail_no_handle(TSD_E_INVALID_ARG, "cache: k_dev, v_dev and page_table_dev must not be NULL");
  if (c->dtype != TSD_F32 && c->dtype != TSD_BF16) return fail_no_handle(TSD_E_INVALID_ARG, "cache: dtype must be TSD_F32 or TSD_BF16");
  if (c->page_tokens < 1 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)))
    return fail_no_handle(TSD_E_INVALID_ARG, "cache: page_tokens must be a power of two, 1..1024");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return fail_no_handle(TSD_E_INVALID_ARG, "cache: n_kv_heads must be 1..1024");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return fail_no_handle(TSD_E_INVALID_ARG, "cache: head_dim must be a multiple of 8, 8..256");
  if (c->n_pages < 1 || c->pages_per_seq < 1 || c->table_stride < c->pages_per_seq)
    return fail_no_handle(TSD_E_INVALID_ARG, "cache: need n_pages >= 1, pages_per_seq >= 1 and table_stride >= pages_per_seq");
  if ((int64_t)c->pages_per_seq * c->page_tokens > INT32_MAX / 2)
    return fail_no_handle(TSD_E_OUT_OF_RANGE, "cache: more than 2^30 tokens per sequence");
  const int es = type_bytes(c->dtype);
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return fail_no_handle(TSD_E_INVALID_ARG, "cache: strides must not be negative");
  if (((c->page_stride | c->token_stride | c->head_stride) * es & 15) || ((reinterpret_cast<uintptr_t>(c->k_dev) | reinterpret_cast<uintptr_t>(c->v_dev)) & 15))
    return fail_no_handle(TSD_E_INVALID_ARG, "cache: the pools and their strides must be multiples of 16 bytes");
  return TSD_OK;
}

int check_rows(const tsd_rows* r, int es, const char* name) {
  if (!r || !r->data_dev) return fail_no_handle(TSD_E_INVALID_ARG, std::string(name) + " must not be NULL");
  if (r->stride_b < 0 || r->stride_t < 0 || r->stride_h < 0) return fail_no_handle(TSD_E_INVALID_ARG, std::string(name) + ": strides must not be negative");
  if (!rows_aligned(*r, es)) return fail_no_handle(TSD_E_INVALID_ARG, std::string(name) + ": data and strides must be multiples of 16 bytes");
  return TSD_OK;
}

PagedView cache_view(const tsd_paged_cache& c) {
  int shift = 0;
  while ((1 << shift) < c.page_tokens) ++shift;
  return {static_cast<char*>(c.k_dev), static_cast<char*>(c.v_dev), (long)c.page_stride, (long)c.token_stride, (long)c.head_stride,
          c.page_table_dev, c.table_stride, c.pages_per_seq, c.n_pages, shift};
}

}  // namespace tsd

using namespace tsd;

extern "C" int tsd_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, int32_t original_len, double low, double high,
                                    double* freq_host, double* amplitude_host) {
  if (!freq_host || !amplitude_host) return fail_no_handle(TSD_E_INVALID_ARG, "freq_host and amplitude_host must not be NULL");
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 256) return fail_no_handle(TSD_E_INVALID_ARG, "rotary_dim must be even, 2..256");
  if (!(base > 1.0) || !std::isfinite(base)) return fail_no_handle(TSD_E_INVALID_ARG, "base must be above 1");
  if (scaling < TSD_ROPE_PLAIN || scaling > TSD_ROPE_BLEND) return fail_no_handle(TSD_E_INVALID_ARG, "scaling: unknown kind");
  if (scaling != TSD_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return fail_no_handle(TSD_E_INVALID_ARG, "factor must be at least 1");
  if (scaling == TSD_ROPE_BASE && rotary_dim < 4) return fail_no_handle(TSD_E_INVALID_ARG, "a stretched base needs rotary_dim >= 4");
  if (scaling == TSD_ROPE_BLEND && (original_len < 1 || !(low < high) || !(low >= 0.0) || !std::isfinite(high)))
    return fail_no_handle(TSD_E_INVALID_ARG, "blended frequencies need original_len >= 1 and 0 <= low < high");
  const int R = rotary_dim;
  if (scaling == TSD_ROPE_BASE) base *= std::pow(factor, (double)R / (R - 2));
  for (int i = 0; i < R / 2; ++i) {
    double f = std::pow(base, -2.0 * i / R);
    if (scaling == TSD_ROPE_LINEAR) f /= factor;
    if (scaling == TSD_ROPE_BLEND) {
      const double turns = original_len * f / (2.0 * M_PI);
      const double keep = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
      f *= keep + (1.0 - keep) / factor;
    }
    freq_host[i] = f;
  }
  *amplitude_host = scaling == TSD_ROPE_BLEND ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return TSD_OK;
}
