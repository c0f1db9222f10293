// mxp_cache_write, mxp_cache_read: rows of keys and values to and from the pages of a quantized cache (layout: mxp_cache.h).
//
// HBM-bound streaming kernels: 2 bytes in and 0.5625 out per bf16 value, or the reverse.  Four lanes share a block, as in the
// dense conversions, with the same arithmetic; what differs is where a row lies: the slot of its token.  A workgroup takes the keys or
// the values of one head of 16 consecutive tokens (D = 128): 256-byte runs of the source, and in the cache, where consecutive tokens
// have consecutive slots, whole lines of one record, scales included (16 rows of one token, whose records lie apart: a tenth slower).
// Which head is the workgroup's, from its place in the grid: a 64-bit division and products per lane cost as much issue time as the
// conversion itself (write 23.4, read 19.1 us below).
// 16384 tokens, 8 heads of 128, bf16, MXFP4+, 86 MB: write 19.9 us (4.3 TB/s), read 15.6 us (5.5 TB/s), with slots at random 20.9 and
// 15.9; 64 tokens 4.6 us, of which a launch alone is 2.3.
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

// A lane's token, its slot and its group of 8 values in a row, for the tile of consecutive tokens that a workgroup takes.
struct Place {
  int64_t token, page;
  int row, group;
  bool there, held;                                          // a token of the call; its slot is in the cache
  __device__ __forceinline__ Place(const CacheRows& a, int64_t tile) {
    const int lanes = a.g.D >> 3;
    token = tile * (256 / lanes) + (int)threadIdx.x / lanes;
    group = (int)threadIdx.x & (lanes - 1);
    there = token < a.tokens;
    const int64_t slot = there ? a.slots[token] : -1;
    page = slot >> a.g.page_shift;
    row = (int)slot & ((1 << a.g.page_shift) - 1);
    held = slot >= 0 && page < a.g.n_pages;
  }
};

// Which rows of the tokens: the keys' (which < kv_heads) or the values' of a head; the same for all lanes.
struct Which {
  int head, is_v;
  __device__ __forceinline__ Which(const CacheRows& a, int which) : head(which < a.g.kv_heads ? which : which - a.g.kv_heads), is_v(which >= a.g.kv_heads) {}
  __device__ __forceinline__ int64_t value(const CacheRows& a, const Place& p) const { return p.token * (is_v ? a.ld_v : a.ld_k) + (head * a.g.D + p.group * 8); }
  __device__ __forceinline__ uint8_t* record(const CacheRows& a, const Place& p) const {
    return a.data + p.page * ((int64_t)a.g.kv_heads * 2 * a.g.part_bytes) + (int64_t)(2 * head + is_v) * a.g.part_bytes;
  }
};

// Groups per lane, U, with their loads under way together: kCacheUnroll where there are rows enough (see cache_unroll), else one.
// blockIdx.x: heads of keys and values, U at a time; blockIdx.y: tiles of tokens.
template <bool BF16, int MODE, int U>
__global__ void __launch_bounds__(256) cache_quantize_kernel(const CacheRows a, int64_t tiles) {
  const int part = threadIdx.x & 3;
  for (int64_t tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
    const Place p(a, tile);
    uint32_t w[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[u][i] = 0;
      if (p.held) {
        const Which x(a, (int)blockIdx.x * U + u);
        const void* src = x.is_v ? a.v : a.k;
        if (BF16) {
          const u32x4 t = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(src) + x.value(a, p)));
          w[u][0] = t.x; w[u][1] = t.y; w[u][2] = t.z; w[u][3] = t.w;
        } else {
          const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(src) + x.value(a, p));
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
      if (p.held) {
        uint8_t* rec = Which(a, (int)blockIdx.x * U + u).record(a, p);
        *reinterpret_cast<uint32_t*>(rec + p.row * (a.g.D >> 1) + p.group * 4) = packed;
        if (part == 0) {
          const int b = p.row * (a.g.D >> 5) + (p.group >> 2);
          rec[a.g.scales_at + b] = (uint8_t)sbyte;
          if (MODE >= 1) rec[a.g.index_at + b] = (uint8_t)idx;
        }
      }
    }
  }
}

template <bool BF16, int MODE, int U>
__global__ void __launch_bounds__(256) cache_dequantize_kernel(const CacheRows a, void* k, void* v, int64_t tiles) {
  const uint32_t part = threadIdx.x & 3u;
  for (int64_t tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
    const Place p(a, tile);
    uint32_t dw[U], sbyte[U], ib[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      dw[u] = sbyte[u] = ib[u] = 0;                          // (scale byte 0: zeros)
      if (p.held) {
        const uint8_t* rec = Which(a, (int)blockIdx.x * U + u).record(a, p);
        const int b = p.row * (a.g.D >> 5) + (p.group >> 2);
        dw[u] = *reinterpret_cast<const uint32_t*>(rec + p.row * (a.g.D >> 1) + p.group * 4);
        sbyte[u] = rec[a.g.scales_at + b];
        if (MODE >= 1) ib[u] = rec[a.g.index_at + b];
      }
    }
    if (!p.there) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t out[8];
      decode_group<(MODE >= 1), BF16>(dw[u], sbyte[u], MODE >= 1 ? ib[u] & 31u : 64u, part, out, MODE == 2 ? ib[u] >> 5 : 0u);
      const Which x(a, (int)blockIdx.x * U + u);
      void* dst = x.is_v ? v : k;
      if (BF16) {
        __builtin_nontemporal_store(u32x4{out[0], out[1], out[2], out[3]}, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + x.value(a, p)));
      } else {
        u32x4* o = reinterpret_cast<u32x4*>(static_cast<float*>(dst) + x.value(a, p));
        o[0] = u32x4{out[0], out[1], out[2], out[3]};        // (half of every line each: 65536 tokens, 2 heads of 64: streaming stores
        o[1] = u32x4{out[4], out[5], out[6], out[7]};        // 26.2 us, these 17.7)
      }
    }
  }
}

// arguments of both directions; on MXP_OK with tokens > 0, `a` and the number of tiles of tokens
int check_rows(const void* k, const void* v, int dtype, int64_t tokens, int64_t ld_k, int64_t ld_v, const int64_t* slots, const void* cache,
               int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt, CacheRows& a, int64_t& tiles) {
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
  tiles = (tokens + rows_per_wg - 1) / rows_per_wg;
  return MXP_OK;
}

// Two groups per lane once that leaves eight workgroups per compute unit.  8 heads of 128, bf16, MXFP4+, one | two | four groups: 16384
// tokens: write 25.2 | 19.9 | 19.8 us, slots at random 26.1 | 20.9 | 22.1, read 18.3 | 15.6 | 17.2; 4096 tokens, the first with two:
// write 9.0 | 7.7, read 6.9 | 6.5.
constexpr int kCacheUnroll = 2;                              // (divides the keys' and values' heads)
bool cache_unroll(const CacheRows& a, int64_t tiles) { return tiles * 2 * a.g.kv_heads >= (int64_t)kNumCU * 8 * kCacheUnroll; }
dim3 grid_of(const CacheRows& a, int64_t tiles) {
  return dim3((unsigned)(cache_unroll(a, tiles) ? 2 * a.g.kv_heads / kCacheUnroll : 2 * a.g.kv_heads), (unsigned)(tiles < 65535 ? tiles : 65535));
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
  int64_t tiles = 0;
  const int rc = check_rows(K, V, src_dtype, tokens, ld_k, ld_v, slots, cache, n_pages, page_tokens, kv_heads, head_dim, fmt, a, tiles);
  if (rc != MXP_OK || tokens == 0) return rc;
  const dim3 grid = grid_of(a, tiles), block(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_WRITE(B, M)                                                                                            \
  do {                                                                                                             \
    if (cache_unroll(a, tiles)) hipLaunchKernelGGL((cache_quantize_kernel<B, M, kCacheUnroll>), grid, block, 0, s, a, tiles); \
    else hipLaunchKernelGGL((cache_quantize_kernel<B, M, 1>), grid, block, 0, s, a, tiles);                         \
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
  int64_t tiles = 0;
  const int rc = check_rows(K, V, dst_dtype, tokens, ld_k, ld_v, slots, cache, n_pages, page_tokens, kv_heads, head_dim, fmt, a, tiles);
  if (rc != MXP_OK || tokens == 0) return rc;
  const dim3 grid = grid_of(a, tiles), block(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_READ(B, M)                                                                                             \
  do {                                                                                                             \
    if (cache_unroll(a, tiles)) hipLaunchKernelGGL((cache_dequantize_kernel<B, M, kCacheUnroll>), grid, block, 0, s, a, K, V, tiles); \
    else hipLaunchKernelGGL((cache_dequantize_kernel<B, M, 1>), grid, block, 0, s, a, K, V, tiles);                 \
  } while (0)
  if (dst_dtype == MXP_BF16) { if (fmt == 0) MXP_READ(true, 0); else if (fmt == 1) MXP_READ(true, 1); else MXP_READ(true, 2); }
  else                       { if (fmt == 0) MXP_READ(false, 0); else if (fmt == 1) MXP_READ(false, 1); else MXP_READ(false, 2); }
#undef MXP_READ
  return launch_status();
}
