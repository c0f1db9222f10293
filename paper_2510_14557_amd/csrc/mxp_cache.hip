// mxp_cache_write, mxp_cache_read: rows of keys and values to and from the pages of a quantized cache (layout: mxp_cache.h).
//
// HBM-bound streaming kernels: 2 bytes in and 0.5625 out per bf16 value, or the reverse.  Four lanes share a block, as in the
// dense conversions, with the same arithmetic; what differs is where a row lies: the slot of its token.  A workgroup takes the keys or
// the values of one head of 16 consecutive tokens (D = 128): 256-byte runs of the source, and in the cache, where consecutive tokens
// have consecutive slots, whole lines of one record, scales included (with 16 rows of one token, whose records lie apart, the write
// below took 26.6 us and the read 20.9).
// 16384 tokens, 8 heads of 128, bf16, MXFP4+, 86 MB: write 23.4 us (3.7 TB/s), read 19.1 us (4.5 TB/s), also with slots at random
// (23.8 | 19.2); 64 tokens 4.8 us, of which a launch alone is 2.3.
#include "mxp_cache.h"
#include "mxp_decode.h"
#include "mxp_encode.h"

namespace {

using namespace mxp;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct CacheRows {
  const void *k, *v;                   // [tokens][kv_heads][D], row strides in elements
  int64_t ld_k, ld_v;
  const int64_t* slots;
  uint8_t* data;
  int64_t tokens;
  CacheGeom g;
};

// One lane's group of 8 values: its row and where the row's record is.  False past the last row.
struct Place {
  int64_t token, slot;
  int head, is_v, group;
  __device__ __forceinline__ bool find(const CacheRows& a, int64_t wg) {
    const int lanes = a.g.D >> 3, rows = 256 / lanes, per = 2 * a.g.kv_heads;
    const int64_t tile = wg / per;                                    // (uniform)
    const int y = (int)(wg - tile * per);
    token = tile * rows + (int)threadIdx.x / lanes;
    is_v = y >= a.g.kv_heads;
    head = y - (is_v ? a.g.kv_heads : 0);
    group = (int)threadIdx.x & (lanes - 1);
    if (token >= a.tokens) return false;
    slot = a.slots[token];
    return true;
  }
  __device__ __forceinline__ bool held(const CacheRows& a) const { return slot >= 0 && (slot >> a.g.page_shift) < a.g.n_pages; }
  __device__ __forceinline__ uint8_t* record(const CacheRows& a) const {
    return a.data + (((slot >> a.g.page_shift) * a.g.kv_heads + head) * 2 + is_v) * a.g.part_bytes;
  }
  __device__ __forceinline__ int row(const CacheRows& a) const { return (int)(slot & ((1 << a.g.page_shift) - 1)); }
  __device__ __forceinline__ int64_t value(const CacheRows& a) const {
    return token * (is_v ? a.ld_v : a.ld_k) + (int64_t)head * a.g.D + group * 8;
  }
};

// Groups per lane, U, with their loads under way together: kCacheUnroll where there are rows enough (see cache_unroll), else one.
template <bool BF16, int MODE, int U>
__global__ void __launch_bounds__(256) cache_quantize_kernel(const CacheRows a, int64_t n_wg) {
  const int part = threadIdx.x & 3;
  for (int64_t wg = (int64_t)blockIdx.x * U; wg < n_wg; wg += (int64_t)gridDim.x * U) {
    Place p[U];
    bool there[U];
    uint32_t w[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) there[u] = p[u].find(a, wg + u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      there[u] = there[u] && p[u].held(a);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[u][i] = 0;
      if (there[u]) {
        const void* src = p[u].is_v ? a.v : a.k;
        if (BF16) {
          const u32x4 t = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(src) + p[u].value(a)));
          w[u][0] = t.x; w[u][1] = t.y; w[u][2] = t.z; w[u][3] = t.w;
        } else {
          const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(src) + p[u].value(a));
          const u32x4 t0 = __builtin_nontemporal_load(q), t1 = __builtin_nontemporal_load(q + 1);
          w[u][0] = t0.x; w[u][1] = t0.y; w[u][2] = t0.z; w[u][3] = t0.w;
          w[u][4] = t1.x; w[u][5] = t1.y; w[u][6] = t1.z; w[u][7] = t1.w;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t sbyte, idx;
      const uint32_t packed = encode_group<BF16, MODE>(w[u], part, sbyte, idx);   // (every lane: the quad exchanges)
      if (there[u]) {
        uint8_t* rec = p[u].record(a);
        const int row = p[u].row(a);
        *reinterpret_cast<uint32_t*>(rec + row * (a.g.D >> 1) + p[u].group * 4) = packed;
        if (part == 0) {
          const int b = row * (a.g.D >> 5) + (p[u].group >> 2);
          rec[a.g.scales_at + b] = (uint8_t)sbyte;
          if (MODE >= 1) rec[a.g.index_at + b] = (uint8_t)idx;
        }
      }
    }
  }
}

template <bool BF16, int MODE, int U>
__global__ void __launch_bounds__(256) cache_dequantize_kernel(const CacheRows a, void* k, void* v, int64_t n_wg) {
  const uint32_t part = threadIdx.x & 3u;
  for (int64_t wg = (int64_t)blockIdx.x * U; wg < n_wg; wg += (int64_t)gridDim.x * U) {
    Place p[U];
    bool there[U];
    uint32_t dw[U], sbyte[U], ib[U];
#pragma unroll
    for (int u = 0; u < U; ++u) there[u] = p[u].find(a, wg + u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      dw[u] = sbyte[u] = ib[u] = 0;                          // (scale byte 0: zeros)
      if (there[u] && p[u].held(a)) {
        const uint8_t* rec = p[u].record(a);
        const int row = p[u].row(a), b = row * (a.g.D >> 5) + (p[u].group >> 2);
        dw[u] = *reinterpret_cast<const uint32_t*>(rec + row * (a.g.D >> 1) + p[u].group * 4);
        sbyte[u] = rec[a.g.scales_at + b];
        if (MODE >= 1) ib[u] = rec[a.g.index_at + b];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      uint32_t out[8];
      decode_group<(MODE >= 1), BF16>(dw[u], sbyte[u], MODE >= 1 ? ib[u] & 31u : 64u, part, out, MODE == 2 ? ib[u] >> 5 : 0u);
      void* dst = p[u].is_v ? v : k;
      if (BF16) {
        __builtin_nontemporal_store(u32x4{out[0], out[1], out[2], out[3]}, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + p[u].value(a)));
      } else {
        u32x4* o = reinterpret_cast<u32x4*>(static_cast<float*>(dst) + p[u].value(a));
        o[0] = u32x4{out[0], out[1], out[2], out[3]};        // (half of every line each: 65536 tokens, 2 heads of 64: streaming stores
        o[1] = u32x4{out[4], out[5], out[6], out[7]};        // 26.2 us, these 17.7)
      }
    }
  }
}

// arguments of both directions; on MXP_OK with tokens > 0, `a` and the number of workgroups' worth of rows
int check_rows(const void* k, const void* v, int dtype, int64_t tokens, int64_t ld_k, int64_t ld_v, const int64_t* slots, const void* cache,
               int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt, CacheRows& a, int64_t& n_wg) {
  const int rc = cache_geom(n_pages, page_tokens, kv_heads, head_dim, fmt, a.g);
  if (rc != MXP_OK) return rc;
  if (dtype != MXP_F32 && dtype != MXP_BF16) return MXP_ERR_DTYPE;
  if (tokens < 0) return MXP_ERR_SHAPE;
  if (tokens == 0) return MXP_OK;
  if (!k || !v || !slots || !cache) return MXP_ERR_NULL;
  const int64_t row = kv_heads * head_dim, esz = dtype == MXP_BF16 ? 2 : 4;
  if (ld_k < row || ld_v < row || tokens > ((int64_t)1 << 40)) return MXP_ERR_SHAPE;
  if (!aligned16(k) || !aligned16(v) || !aligned16(cache) || (reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || ld_k * esz % 16 != 0 ||
      ld_v * esz % 16 != 0)
    return MXP_ERR_ALIGN;
  const int64_t rows_per_wg = 256 / (head_dim / 8);
  a.k = k;
  a.v = v;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.slots = slots;
  a.data = static_cast<uint8_t*>(const_cast<void*>(cache));
  a.tokens = tokens;
  n_wg = (tokens + rows_per_wg - 1) / rows_per_wg * 2 * kv_heads;
  return MXP_OK;
}

// Two groups per lane once that leaves two rounds of eight workgroups per compute unit.  16384 tokens as above, one | two | four groups:
// write 27.0 | 23.4 | 24.8 us, read 21.0 | 19.1 | 19.4; 4096 tokens, below the rule: one and two alike (9.5).
constexpr int kCacheUnroll = 2;
bool cache_unroll(int64_t n_wg) { return n_wg >= (int64_t)kNumCU * 16 * kCacheUnroll; }
unsigned grid_of(int64_t n_wg) {
  const int64_t n = cache_unroll(n_wg) ? (n_wg + kCacheUnroll - 1) / kCacheUnroll : n_wg;
  return (unsigned)(n < ((int64_t)1 << 23) ? n : ((int64_t)1 << 23));   // (a launch has fewer than 2^32 threads)
}

}  // namespace

extern "C" size_t mxp_cache_bytes(int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt) {
  mxp::CacheGeom g;
  if (mxp::cache_geom(n_pages, page_tokens, kv_heads, head_dim, fmt, g) != MXP_OK) return 0;
  return (size_t)n_pages * (size_t)kv_heads * 2 * (size_t)g.part_bytes;
}

extern "C" int mxp_cache_write(const void* K, const void* V, int src_dtype, int64_t tokens, int64_t ld_k, int64_t ld_v, const int64_t* slots,
                               void* cache, int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt, void* stream) {
  using namespace mxp;
  CacheRows a;
  int64_t n_wg = 0;
  const int rc = check_rows(K, V, src_dtype, tokens, ld_k, ld_v, slots, cache, n_pages, page_tokens, kv_heads, head_dim, fmt, a, n_wg);
  if (rc != MXP_OK || tokens == 0) return rc;
  const dim3 grid(grid_of(n_wg)), block(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_WRITE(B, M)                                                                                            \
  do {                                                                                                             \
    if (cache_unroll(n_wg)) hipLaunchKernelGGL((cache_quantize_kernel<B, M, kCacheUnroll>), grid, block, 0, s, a, n_wg); \
    else hipLaunchKernelGGL((cache_quantize_kernel<B, M, 1>), grid, block, 0, s, a, n_wg);                         \
  } while (0)
  if (src_dtype == MXP_BF16) { if (fmt == 0) MXP_WRITE(true, 0); else if (fmt == 1) MXP_WRITE(true, 1); else MXP_WRITE(true, 2); }
  else                       { if (fmt == 0) MXP_WRITE(false, 0); else if (fmt == 1) MXP_WRITE(false, 1); else MXP_WRITE(false, 2); }
#undef MXP_WRITE
  return launch_status();
}

extern "C" int mxp_cache_read(const void* cache, int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt,
                              const int64_t* slots, int64_t tokens, void* K, void* V, int dst_dtype, int64_t ld_k, int64_t ld_v, void* stream) {
  using namespace mxp;
  CacheRows a;
  int64_t n_wg = 0;
  const int rc = check_rows(K, V, dst_dtype, tokens, ld_k, ld_v, slots, cache, n_pages, page_tokens, kv_heads, head_dim, fmt, a, n_wg);
  if (rc != MXP_OK || tokens == 0) return rc;
  const dim3 grid(grid_of(n_wg)), block(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_READ(B, M)                                                                                             \
  do {                                                                                                             \
    if (cache_unroll(n_wg)) hipLaunchKernelGGL((cache_dequantize_kernel<B, M, kCacheUnroll>), grid, block, 0, s, a, K, V, n_wg); \
    else hipLaunchKernelGGL((cache_dequantize_kernel<B, M, 1>), grid, block, 0, s, a, K, V, n_wg);                 \
  } while (0)
  if (dst_dtype == MXP_BF16) { if (fmt == 0) MXP_READ(true, 0); else if (fmt == 1) MXP_READ(true, 1); else MXP_READ(true, 2); }
  else                       { if (fmt == 0) MXP_READ(false, 0); else if (fmt == 1) MXP_READ(false, 1); else MXP_READ(false, 2); }
#undef MXP_READ
  return launch_status();
}
