// Geometry of the paged key-value cache, shared by the kernels that write, read and attend over it.
//
// A page holds page_tokens tokens.  For each key-value head it holds a record of the keys and, behind it, one of the values:
//     [page_tokens][D / 2] codes | [page_tokens][D / 32] scale bytes | [page_tokens][D / 32] index bytes (not for MXFP4)
// that is, a small canonical operand whose blocks run along the head.  All that a head's attention reads of a page is one
// contiguous run (16 tokens of D = 128: 2304 bytes), so a wavefront that takes a page of one head moves whole lines only.
#pragma once
#include "mxp_common.h"

namespace mxp {

struct CacheGeom {
  int64_t n_pages;
  int page_shift, kv_heads, D;         // page_tokens = 1 << page_shift
  int scales_at, index_at, part_bytes; // offsets in a record, its size
};

inline bool cache_format(int fmt) { return fmt >= MXP_FMT_MXFP4 && fmt <= MXP_FMT_MXFP4PP; }

// MXP_OK and the geometry, or what is wrong with it
inline int cache_geom(int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt, CacheGeom& g) {
  if (!cache_format(fmt)) return fmt >= 0 && fmt <= MXP_FMT_MXFP8P ? MXP_ERR_UNSUPPORTED : MXP_ERR_FORMAT;
  if (n_pages < 1 || n_pages > 2147483647LL || kv_heads < 1 || kv_heads > 65535 || page_tokens < 1 || head_dim < 1) return MXP_ERR_SHAPE;
  if (page_tokens < 16 || page_tokens > 256 || (page_tokens & (page_tokens - 1)) || (head_dim != 64 && head_dim != 128 && head_dim != 256))
    return MXP_ERR_UNSUPPORTED;
  g.n_pages = n_pages;
  g.page_shift = __builtin_ctzll((unsigned long long)page_tokens);
  g.kv_heads = (int)kv_heads;
  g.D = (int)head_dim;
  g.scales_at = (int)(page_tokens * head_dim / 2);
  g.index_at = g.scales_at + (int)(page_tokens * head_dim / kBlock);
  g.part_bytes = g.index_at + (fmt == MXP_FMT_MXFP4 ? 0 : (int)(page_tokens * head_dim / kBlock));
  return MXP_OK;
}

}  // namespace mxp
