// mxp_attention: softmax attention of ragged query rows over the paged four-bit cache (layout: mxp_cache.h).
//
// One pass over the visible tokens with the running maximum and sum of the softmax, in base 2 (the scale carries log2 e):
//     S = K Q^T     m' = max(m, S)     P = 2^(S - m')     l = l 2^(m - m') + sum P     O = O 2^(m - m') + V^T P     (m: see kGrowth)
// Both products have the tokens' side as their first operand, so the result of the first, [token][row], has a query row per lane
// column and four or sixteen tokens in a lane's registers: what the second takes as its second operand, up to a permutation of the
// tokens inside one MFMA step, which the reads of V follow.  Maximum, sum and rescaling are then a lane's own business (plus one
// exchange between the lanes of a column), and P never leaves the registers.
//
// Keys and values are de-converted (Eq. 2, exact in bf16) into LDS, a lane per block: 16 unpack-converts, four 16-byte stores, and
// the block maximum of a + format as one 2-byte store over its element (30 vector instructions less than merging it in registers).  V
// is read back transposed by the LDS hardware (4 tokens x 16 channels per 16 lanes).
//
// Query rows of one key-value head (heads that share it x queries) are taken together.  attn_few_kernel: up to 32 of them per
// workgroup, every wavefront with tokens of its own, joined through LDS at the end; bound by reading the cache (64 sequences of 2048 to
// 8192 tokens, 8 heads of 128, 32 query heads, MXFP4+: 90 us = 4.2 TB/s with the join's 5 us; of 8192 each 4.7, plain MXFP4 5.2, with
// 64 query heads and pages of 64 5.5; the loads alone 78 us of the 90; vector ALU 66 %, LDS 60 %, matrix cores 12 % of the time).
// attn_many_kernel: 128 rows per workgroup, the wavefronts share the de-converted tokens; bound by the softmax's vector instructions and
// the matrix cores in turn (one prompt of 8192 tokens, 32 heads of 128 on 8: 600 to 627 us on several machines = 877 to 916 TFLOP/s;
// vector ALU 56 %, matrix cores 39 %, LDS 35 %; the next tile's scores formed among this one's weights: 3 % slower, the registers do
// not hold both).  At head_dim 256 the registers do not hold a wavefront's rows either: 31 to 52 a lane lie in scratch memory (a prompt
// of 2048 tokens 193 us = 356 TFLOP/s).
// Both can deal a sequence's tokens out to several workgroups; attn_join_kernel then joins the parts.
#include "mxp_cache.h"

namespace {

using namespace mxp;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4), may_alias));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16a __attribute__((may_alias));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4), may_alias));
typedef float f32x16 __attribute__((ext_vector_type(16)));

union Operand {                                              // eight bf16 of an MFMA operand
  uint32_t u[4];
  s16x4 s[2];
  bf16x8 v;
};

struct AttnArgs {
  const uint16_t* q;
  int64_t ld_q, rows;
  const int32_t *q_start, *kv_len, *table;
  int64_t ld_table;
  int n_seq, heads, group, causal, window;                   // group: query heads per key-value head; window 0: none
  float scale, up;                                           // |scale| * log2(e), at least the smallest normal number; kGrowth over it
  uint32_t flip;                                             // sign bits of two bf16 where scale is negative: Q is negated
  const uint8_t* data;
  CacheGeom g;
  void* o;
  int64_t ld_o;
  int o_bf16;
  float *lse, *part_o, *part_ml;                             // parts of rows: D values; what their weights refer to, their sum
  int32_t* joins;                                            // few rows: [workgroup][4], see Share
  int row_tiles;
};

constexpr int kWaves = 4;                                     // of a workgroup
constexpr float kInf = __builtin_inff();
// What a row's weights refer to, m, is set 2^kGrowth above the largest score seen, and again only where a score exceeds it: most tiles of
// tokens need no rescaling, and a weight is never above 1, so that sums of weighted values stay below those of the values.  Weights
// of 2^-kGrowth have the relative error of larger ones in bf16 and in the fp32 sums; below 2^-118 of the row's largest they may count as 0.
constexpr float kGrowth = 8.0f, kMostFloat = 3.40282347e38f;
__device__ __forceinline__ float raised(float m, float mx, float up) { return mx > m ? fminf(mx + up, kMostFloat) : m; }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float zero_if_none(float m) { return m == -kInf ? 0.0f : m; }   // 2^(x - m) where nothing was seen yet

__device__ __forceinline__ float max_across_16(float x) {    // over lanes l, l ^ 16
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float max_across_32(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float sum_across_16(float x) {
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}
__device__ __forceinline__ float sum_across_32(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {   // rounded to nearest even
  union { bf16x2 v; uint32_t u; } c;
  c.v = bf16x2{(__bf16)a, (__bf16)b};
  return c.u;
}

constexpr int64_t kMostTokens = (int64_t)1 << 30, kMostRows = (int64_t)1 << 30;   // per sequence; rows x heads of a call

// Eight weights of one row, 2^(scale x - base), as the bf16 terms of an operand; their sum, of the unrounded ones.  A term is the
// rounded rest that the terms before it leave: three hold all 24 bits, for fp32 results.  bf16 results have one: their relative error
// against 64 bits (norms) is then 2.1e-3 to 2.3e-3, of which the rounding of the results alone is 1.65e-3.  Two terms leave that only, at
// another product per tile of V: the prompt 605 -> 762 us, 64 sequences of one query 89.5 -> 94.
template <int TERMS>
__device__ __forceinline__ float weights(f32x4 x0, f32x4 x1, float scale, float base, Operand (&p)[TERMS]) {
  float e[8], sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = exp2_of(__builtin_fmaf(j < 4 ? x0[j & 3] : x1[j & 3], scale, -base));
#pragma unroll
  for (int j = 0; j < 8; j += 2) sum += e[j] + e[j + 1];
#pragma unroll
  for (int c = 0; c < TERMS; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u = bf16_pair(e[2 * j], e[2 * j + 1]);
      p[c].u[j] = u;
      e[2 * j] -= __uint_as_float(u << 16);
      e[2 * j + 1] -= __uint_as_float(u & 0xFFFF0000u);
    }
  return sum;
}

// a value that all lanes have, where the compiler cannot see it
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// ---- one sequence's share of the work -------------------------------------------------------------------------------
struct Sequence {
  int64_t q0;                                                // first row of Q
  int n, kv;                                                 // queries, tokens in the cache
  const int32_t* pages;
  __device__ __forceinline__ Sequence(const AttnArgs& a, int s) {
    int64_t first = s, end = (int64_t)s + 1;
    if (a.q_start) {
      first = a.q_start[s];
      end = a.q_start[s + 1];
    }
    first = first < 0 ? 0 : first;
    end = end > a.rows ? a.rows : end;
    q0 = first;
    n = end > first ? (int)(end - first) : 0;
    const int64_t table_end = a.ld_table < kMostTokens ? a.ld_table << a.g.page_shift : kMostTokens;
    const int64_t most = table_end < kMostTokens ? table_end : kMostTokens, len = a.kv_len[s];
    kv = (int)(len < 0 ? 0 : len > most ? most : len);
    pages = a.table + s * a.ld_table;
  }
  // tokens [first, last] that query i sees
  __device__ __forceinline__ int last(const AttnArgs& a, int i) const { return a.causal ? kv - n + i : kv - 1; }
  __device__ __forceinline__ int first(const AttnArgs& a, int i) const {
    const int l = kv - n + i;
    return a.window > 0 && l >= a.window ? l - a.window + 1 : 0;
  }
};

// The tokens [first, end) that any of `rows` > 0 rows from `row` on sees (each of them by some row); begin: where the tiles of tokens
// start, a multiple of 32 at most 31 tokens in front of them, or a share's begin.
struct Span {
  int first = 0, begin = 0, end = 0;
  Span() = default;
  __device__ __forceinline__ Span(const AttnArgs& a, const Sequence& s, int row, int rows) {
    first = s.first(a, row / a.group);
    begin = first & ~31;
    end = s.last(a, (row + rows - 1) / a.group) + 1;
  }
};

// how many tokens there are from `first` to `last`, before `end`
__device__ __forceinline__ uint32_t tokens_from_to(int first, int last, int end) {
  const int n = (last < end ? last + 1 : end) - first;
  return n > 0 ? (uint32_t)n : 0u;
}

// The page of a token: its number, or -1 where it has none
__device__ __forceinline__ int32_t page_of(const AttnArgs& a, const Sequence& s, int64_t t) {
  const int64_t j = t >> a.g.page_shift;
  const int32_t p = j < a.ld_table ? s.pages[j] : -1;
  return p < a.g.n_pages ? p : -1;
}
struct Page {
  const uint8_t* rec;                                        // its record of this head's keys (page 0's if there is none)
  int at;                                                    // the token's place in it
  bool held;
  __device__ __forceinline__ Page(const AttnArgs& a, int head, int32_t p, int t) {
    held = p >= 0;
    rec = a.data + ((int64_t)(held ? p : 0) * a.g.kv_heads + head) * 2 * a.g.part_bytes;
    at = t & ((1 << a.g.page_shift) - 1);
  }
};

// ---- a block of 32 values -------------------------------------------------------------------------------------------
struct Block {
  u32x4 code;
  uint32_t scale, index;
  // To be expanded to zeros, as a flushed block is.  For values in front of the first token that any row sees: their slots may never have
  // been written, and weights of 0 do not hide an Inf or NaN.  Only the first tile of a span has such tokens, so they are blanked once,
  // ahead of the loop (tested inside it, the one number more that lives through the loop spills: 64 sequences 89 -> 95 us).
  __device__ __forceinline__ void blank() { scale = index = 0u; }
};

// ONCE: no other workgroup of the call reads these codes (64 sequences of 2048 to 8192 tokens 95.5 -> 89.4 us with streaming loads)
template <int D, int MODE, bool ONCE>
__device__ __forceinline__ Block load_block(const uint8_t* rec, const CacheGeom& g, int row, int blk) {
  Block b;
  const int n = row * (D / 32) + blk;
  const u32x4* const code = reinterpret_cast<const u32x4*>(rec + n * 16);
  b.code = ONCE ? __builtin_nontemporal_load(code) : *code;
  b.scale = rec[g.scales_at + n];
  b.index = MODE >= 1 ? rec[g.index_at + n] : 0u;
  return b;
}

// Tokens in LDS: 2 D bytes each, without gaps, the 16-byte pieces of a token in an order of its own: piece c lies at c ^ s(token).
// With s below the 16 pieces that 16 tokens have at the same channels fall on all banks (the stores of a de-converted block per
// lane, the reads of K), and so do four neighbouring tokens' 64 bytes each (the transposed reads of V); rows padded to a pitch of
// 2 D + 16 bytes left more than half of the LDS cycles to conflicts.  `at` is the token's place, a multiple of 2 D, with its s: the
// piece at channel byte b (a multiple of 16) is at ^ b.
template <int D>
__device__ __forceinline__ uint32_t token_at(int token) {
  const uint32_t t = (uint32_t)token;
  const uint32_t s = D == 64 ? ((t & 2u) << 1) | (((t >> 2) & 3u) ^ ((t & 1u) << 1)) : ((t & 3u) << 2) | (((t >> 2) & 3u) ^ (t & 2u));
  return t * (2u * D) | (s << 4);
}

// A place whose variants (^ b) are to be formed where they are used: kept in registers over the loop, they cost the few-row kernel its
// fourth wavefront per SIMD or spill (64 sequences of 2048 to 8192 tokens: 95.2 us, and 89.4 so; of plain MXFP4, 8192 each: 114, and 109).
__device__ __forceinline__ uint32_t formed_at_use(uint32_t at) {
  asm volatile("" : "+v"(at));
  return at;
}

// A block's 32 bf16 into LDS, its first byte at tile + at (`at` as above, with the block's channels).  A flushed block, or one to be
// left out (`drop`), becomes zeros; a scale byte of 255 makes the unpack-converts answer NaN, also for zero codes, so what is left out
// gets another.  Both go by the scale byte, whatever the index byte says (an NBM scale below 0 counts as 0).
template <int MODE>
__device__ __forceinline__ void expand(const Block& b, bool drop, uint8_t* tile, uint32_t at) {
  const bool zero = drop || b.scale == 0u;
  const uint32_t keep = zero ? 0u : 0xFFFFFFFFu;
  const uint32_t delta = MODE == 2 && b.scale != 255u ? b.index >> 5 : 0u;
  const float X = __uint_as_float((drop ? 127u : __builtin_elementwise_sub_sat(b.scale, delta)) << 23);
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t c = b.code[j] & keep;
    union { bf16x2 v; uint32_t u; } w0, w1, w2, w3;
    w0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0);
    w1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1);
    w2.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2);
    w3.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3);
    *reinterpret_cast<u32x4*>(tile + (at ^ (16u * j))) = u32x4{w0.u, w1.u, w2.u, w3.u};
  }
  if (MODE >= 1) {                                           // 2^e_max * 1.mmm * 2^shared_exp over its element
    const uint32_t pos = b.index & 31u;
    const uint32_t lo = pos & 8u ? b.code[1] : b.code[0], hi = pos & 8u ? b.code[3] : b.code[2];
    const uint32_t nib = ((pos & 16u ? hi : lo) >> (4u * (pos & 7u))) & 15u;
    const uint32_t h = (((nib & 8u) << 12) | ((b.scale + 2u) << 7) | ((nib & 7u) << 4)) & keep;   // (scale byte 255: any number among NaN)
    *reinterpret_cast<u16a*>(tile + (at ^ (2u * pos))) = (uint16_t)h;
  }
}

// A block of plain MXFP4 as four operands of eight, in registers.
__device__ __forceinline__ void expand(const Block& b, Operand (&out)[4]) {
  const float X = __uint_as_float(b.scale << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t c = b.scale == 0u ? 0u : b.code[j];
    union { bf16x2 v; uint32_t u; } w0, w1, w2, w3;
    w0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0);
    w1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1);
    w2.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2);
    w3.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3);
    out[j].u[0] = w0.u;
    out[j].u[1] = w1.u;
    out[j].u[2] = w2.u;
    out[j].u[3] = w3.u;
  }
}

// four tokens x 16 channels per 16 lanes, transposed: a lane gets four tokens of one channel
__device__ __forceinline__ s16x4 read_transposed(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t row, int head, int d, f32x4 v) {
  const int64_t off = row * a.ld_o + (int64_t)head * a.g.D + d;
  if (a.o_bf16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + off) = u32x2{bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + off) = v;
}

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f; }
// The end of a row: the output itself, or a part of it
__device__ __forceinline__ void finish_values(const AttnArgs& a, int64_t part_row, int64_t row, int head, int d, f32x4 v, float l) {
  if (part_row < 0) store_out(a, row, head, d, l == 0.0f ? f32x4{0, 0, 0, 0} : v / l);
  else *reinterpret_cast<f32x4*>(a.part_o + part_row * a.g.D + d) = v;
}
__device__ __forceinline__ void finish_row(const AttnArgs& a, int64_t part_row, int64_t row, int head, float m, float l) {
  if (part_row >= 0) {
    a.part_ml[2 * part_row] = m;
    a.part_ml[2 * part_row + 1] = l;
  } else if (a.lse) {
    a.lse[row * a.heads + head] = lse_of(m, l);
  }
}

// ---- dealing out the work --------------------------------------------------------------------------------------------
// How a call's work is dealt to workgroups where it is split: in units of tokens, counted over sequences, their key-value heads and
// their tiles of rows.  A workgroup's share, g of n, is units [g total / n, (g + 1) total / n), whatever the lengths are: it may begin
// and end inside a tile of rows.  Those two leave parts in the workspace, at 2 g (begun by another share) and 2 g + 1 (begun in this
// one); what lies between them is finished here.  The share that begins rows that others go on with records so, and
// attn_join_kernel adds its part and those of the shares behind it.
struct Load {
  int first, end, units, tiles;                              // tokens that any row sees, in units; tiles of rows
  int64_t total;                                             // units x tiles x key-value heads
  __device__ __forceinline__ Load(const AttnArgs& a, const Sequence& s, int rows, int unit) {
    first = end = 0;
    if (s.n > 0) {
      first = s.first(a, 0) & ~31;
      end = s.last(a, s.n - 1) + 1;
    }
    units = end > first ? (end - first + unit - 1) / unit : 1;   // (rows that see nothing are written too)
    tiles = (s.n * a.group + rows - 1) / rows;
    total = (int64_t)units * tiles * a.g.kv_heads;
  }
};
// Shares of so many units, each at least `least`, or half of that while they are fewer than the compute units (one sequence of 2048
// tokens, 8 heads: 17.0 us with four, 14.8 with two; 16 such sequences 22.3 with four, 26.1 with two).
__host__ __device__ inline int64_t shares_of(int64_t units, int64_t least) {
  const int64_t n = (units + least - 1) / least, twice = (units + least / 2 - 1) / (least / 2);
  return n >= kNumCU ? n : twice < kNumCU ? twice : kNumCU;
}
struct Share {
  int64_t begin, end, total;                                 // this workgroup's units; all
  int seq, item, off, n, me;                                 // where `begin` is: sequence, item in it, unit of the item; shares; the number of this one
  __device__ __forceinline__ int workgroup_of(int64_t unit) const { return (int)(((unit + 1) * n - 1) / total); }
};
__device__ __forceinline__ void find_share(const AttnArgs& a, int rows, int unit, int least, bool near, Share& share, int64_t (&wave_sum)[kWaves]) {
  const int each = (a.n_seq + 64 * kWaves - 1) / (64 * kWaves), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s0 = (int)threadIdx.x * each, s1 = s0 + each < a.n_seq ? s0 + each : a.n_seq;
  int64_t mine = 0;
  for (int s = s0; s < s1; ++s) mine += Load(a, Sequence(a, s), rows, unit).total;
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    upto += lane >= d ? x : 0;
  }
  if (lane == 63) wave_sum[wave] = upto;
  if (threadIdx.x == 0) {                                    // (what a workgroup without a share finds)
    share.begin = share.end = share.total = 0;
    share.seq = share.item = share.off = share.n = 0;
  }
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) upto += wave_sum[w];
    total += wave_sum[w];
  }
  const int64_t most = shares_of(total, least), n = most < (int64_t)gridDim.x ? most : (int64_t)gridDim.x;
  // near: neighbouring shares, which then often read the same tokens, on one XCD (workgroups go to the eight of them in turn).  Chunks
  // behind long contexts 151.8 -> 148.4 us; few rows, whose tokens nobody else reads, gain nothing by it.
  const int64_t eights = near ? n >> 3 : 0, id = blockIdx.x, g = id < 8 * eights ? (id & 7) * eights + (id >> 3) : id;
  if (threadIdx.x == 0) share.me = (int)g;
  if (g < n) {
    const int64_t begin = g * total / n, end = (g + 1) * total / n;
    int64_t before = upto - mine;
    if (begin >= before && begin < upto)                     // one lane: the sequence is one of its own
      for (int s = s0; s < s1; ++s) {
        const Load load(a, Sequence(a, s), rows, unit);
        if (begin < before + load.total) {
          share.begin = begin;
          share.end = end;
          share.total = total;
          share.seq = s;
          share.item = (int)((begin - before) / load.units);
          share.off = (int)((begin - before) % load.units);
          share.n = (int)n;
          break;
        }
        before += load.total;
      }
  }
  __syncthreads();
}

// The rows and tokens that a workgroup goes over, one run after another: its share, or (DIRECT) whole tiles of rows.  Two kernels, not a
// branch in one: with the code of both, a prompt of 500 tokens took 24.0 us instead of 21.6, one of 8192 tokens 627 instead of 608.
template <bool DIRECT>
struct Walk {
  int seq, kv_head = 0, tile = 0, item = 0, off = 0, me = 0;
  int64_t left = 0, end = 0;
  int part = -1;                                             // where a run's result goes: out, or among the parts
  __device__ __forceinline__ Walk(const AttnArgs& a, int rows, int unit, int least, bool near, Share& share, int64_t (&wave_sum)[kWaves]) {
    if constexpr (DIRECT) {
      // key-value head fastest (consecutive workgroups go to different XCDs: with 8 heads an XCD's cache has one to hold), then tile
      // of rows, the longest first, then sequence
      uint32_t id = blockIdx.x;
      kv_head = (int)(id % (uint32_t)a.g.kv_heads);
      id /= (uint32_t)a.g.kv_heads;
      tile = (int)(id % (uint32_t)a.row_tiles);
      seq = (int)(id / (uint32_t)a.row_tiles);
    } else {
      find_share(a, rows, unit, least, near, share, wave_sum);
      me = uniform(share.me);
      if (threadIdx.x == 0) a.joins[4 * me] = -1;
      end = uniform(share.end);
      left = end - uniform(share.begin);
      seq = uniform(share.seq);
      item = uniform(share.item);
      off = uniform(share.off);
    }
  }
  // whether there is more to do; `seq` is a sequence's number only then
  __device__ __forceinline__ bool more(const AttnArgs& a) const { return DIRECT || (left > 0 && seq < a.n_seq); }
  __device__ __forceinline__ bool more(const AttnArgs& a, const Sequence& s, int rows) const { return !DIRECT || tile * rows < s.n * a.group; }
  // The next run: its tile of rows and span of tokens.  False where the sequence has none left (the next one may).
  __device__ __forceinline__ bool next(const AttnArgs& a, const Sequence& s, int rows, int unit, const Share& share, int& r0, Span& span) {
    const int R = s.n * a.group;
    int from = 0, to = 0x7FFFFFFF;
    if constexpr (DIRECT) {
      const int tiles = (R + rows - 1) / rows;
      r0 = (tiles - 1 - tile) * rows;                        // the last rows see most: they start first
      tile += a.row_tiles;
    } else {
      const Load load(a, s, rows, unit);
      if (item >= load.tiles * a.g.kv_heads) {
        ++seq;
        item = 0;
        return false;
      }
      const int till = left < load.units - off ? off + (int)left : load.units;
      kv_head = item / load.tiles;
      r0 = (item - kv_head * load.tiles) * rows;
      from = load.first + off * unit;
      if (till < load.units) to = load.first + till * unit;
      part = -1;
      if (off > 0 || till < load.units) {
        part = 2 * me + (off == 0 ? 1 : 0);
        if (off == 0 && threadIdx.x == 0) {                  // the first part of these rows: the join goes on to the last one's workgroup
          int32_t* const j = a.joins + 4 * me;
          j[1] = kv_head;
          j[2] = r0;
          j[3] = share.workgroup_of(end - left + load.units - 1);
          j[0] = seq;
        }
      }
      left -= till - off;
      off = 0;
      ++item;
    }
    span = Span(a, s, r0, R - r0 < rows ? R - r0 : rows);
    if (span.begin < from) span.begin = from;
    if (span.end > to) span.end = to;
    return true;
  }
};

// ---- joining parts --------------------------------------------------------------------------------------------------
// One row of one head from its parts, by a workgroup: every lane the weights of some parts, then D / 4 lanes across a row and
// 1024 / D parts at a time.
constexpr int kMostParts = 1024;
constexpr float kLeftOut = -1.0f;                            // weight of a part that saw nothing (not 0: a NaN of a part too small to count counts)
struct JoinRoom {
  float weight[kMostParts], top_of[4], sum_of[4];
  __attribute__((aligned(16))) float acc[1024];
};
template <class PartAt>
__device__ __forceinline__ void join_row(const AttnArgs& a, JoinRoom& room, int parts, PartAt part_at, int64_t row, int head) {
  const int t = threadIdx.x, across = a.g.D >> 2, d = 4 * (t & (across - 1)), g = t / across, groups = 256 / across;
  float m[kMostParts / 256], l[kMostParts / 256], top = -kInf, sum = 0.0f;
#pragma unroll
  for (int k = 0; k < kMostParts / 256; ++k) {
    m[k] = -kInf;
    l[k] = 0.0f;
    if (t + 256 * k < parts) {
      const int64_t at = part_at(t + 256 * k);
      m[k] = a.part_ml[2 * at];
      l[k] = a.part_ml[2 * at + 1];
    }
    top = fmaxf(top, m[k]);
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  if ((t & 63) == 0) room.top_of[t >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(room.top_of[0], room.top_of[1]), fmaxf(room.top_of[2], room.top_of[3]));
#pragma unroll
  for (int k = 0; k < kMostParts / 256; ++k) {
    const float f = l[k] == 0.0f ? kLeftOut : exp2_of(m[k] - zero_if_none(top));
    room.weight[t + 256 * k] = f;
    if (l[k] != 0.0f) sum += l[k] * f;
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
  if ((t & 63) == 0) room.sum_of[t >> 6] = sum;
  __syncthreads();
  sum = (room.sum_of[0] + room.sum_of[1]) + (room.sum_of[2] + room.sum_of[3]);
  f32x4 out = {0, 0, 0, 0};
  for (int p0 = g; p0 < parts; p0 += 8 * groups) {           // eight loads at a time
    f32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + k * groups;
      x[k] = *reinterpret_cast<const f32x4*>(a.part_o + part_at(p < parts ? p : p0) * a.g.D + d);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + k * groups;
      const float w = p < parts ? room.weight[p] : kLeftOut;
      if (w != kLeftOut) out += x[k] * w;
    }
  }
  *reinterpret_cast<f32x4*>(room.acc + 4 * t) = out;
  __syncthreads();
  if (g == 0) {
    for (int p = 1; p < groups; ++p) out += *reinterpret_cast<const f32x4*>(room.acc + 4 * (t + p * across));
    store_out(a, row, head, d, sum == 0.0f ? f32x4{0, 0, 0, 0} : out / sum);
  }
  if (t == 0 && a.lse) a.lse[row * a.heads + head] = lse_of(top, sum);
  __syncthreads();
}

// The same by a wavefront, for at most 64 parts: a part's weight is a lane's.
template <class PartAt>
__device__ __forceinline__ void join_row_by_wave(const AttnArgs& a, int parts, PartAt part_at, int64_t row, int head) {
  const int lane = threadIdx.x & 63, across = a.g.D >> 2, d = 4 * (lane & (across - 1)), g = lane / across, groups = 64 / across;
  float m = -kInf, l = 0.0f;
  if (lane < parts) {
    const int64_t at = part_at(lane);
    m = a.part_ml[2 * at];
    l = a.part_ml[2 * at + 1];
  }
  f32x4 x[4];                                                // (on their way before the weights are known)
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int p = g + k * groups;
    x[k] = *reinterpret_cast<const f32x4*>(a.part_o + part_at(p < parts ? p : 0) * a.g.D + d);
  }
  float top = m;
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
  const float f = l == 0.0f ? kLeftOut : exp2_of(m - zero_if_none(top));
  float sum = l == 0.0f ? 0.0f : l * f;
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) sum += __shfl_xor(sum, i);
  f32x4 out = {0, 0, 0, 0};
  for (int p0 = 0; p0 < parts; p0 += 4 * groups) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int p = p0 + g + k * groups;
      const float w = __shfl(f, p & 63);
      if (p < parts && w != kLeftOut) out += (p0 == 0 ? x[k] : *reinterpret_cast<const f32x4*>(a.part_o + part_at(p) * a.g.D + d)) * w;
    }
  }
  for (int i = across; i < 64; i <<= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] += __shfl_xor(out[k], i);
  if (g == 0) store_out(a, row, head, d, sum == 0.0f ? f32x4{0, 0, 0, 0} : out / sum);
  if (lane == 0 && a.lse) a.lse[row * a.heads + head] = lse_of(top, sum);
}

// ---- few rows -------------------------------------------------------------------------------------------------------
constexpr int kFewUnit = 32 * kWaves, kFewLeast = 4;          // tokens (a 32-token tile per wavefront); units per workgroup at least
constexpr int kFewAhead = 1;                   // tiles in flight per wavefront
template <int D>
constexpr int few_patch(int nt) { return 64 * D * nt; }      // a tile of 32 tokens (2 D bytes each); 16 nt rows of fp32 for the join
template <int D>
constexpr int few_lds(int nt, int waves) { return waves * (few_patch<D>(nt) + 16 * nt * 8); }
// Wavefronts of a workgroup that has a compute unit to itself.  A tile of tokens takes about 1.6 us there whatever runs beside it (its
// steps wait for one another, more than for memory: tiles fetched two or three ahead change nothing), so more wavefronts are gone
// through sooner, up to what joining them costs: one sequence of 512 | 1024 | 2048 tokens 11.5 | 18.2 | 29.3 us with four, 10.7 | 15.3 |
// 22.2 with eight, 12.4 | 16.7 | 22.0 with sixteen.
// The registers that this leaves do not suffice for 32 rows of head_dim 256, where 25 to 42 a lane lie in scratch memory (64 sequences of
// 2048 to 8192 tokens, 32 query heads on 8: one query 189 us, five 484; at head_dim 128 90 and 127), nor, in workgroups that share,
// for 32 rows of head_dim 64 with fp32 results (9 to 17).
constexpr int few_waves_per_simd(int D, int NT) { return D * NT <= 128 ? 4 : D * NT <= 256 ? 2 : 1; }   // of workgroups that share
constexpr int few_waves_alone(int D, int NT) { return D * NT <= 256 ? 8 : 4; }

// NT tiles of 16 rows; TERMS: bf16 terms of P
template <int D, int MODE, int NT, int TERMS, int WAVES, bool DIRECT>
__global__ void __launch_bounds__(64 * WAVES, WAVES == kWaves ? few_waves_per_simd(D, NT) : WAVES / 4) attn_few_kernel(const AttnArgs a) {
  // A lane's block is, for D >= 128, what the first product wants of its token from it, if its channels are taken in that order: keys
  // of plain MXFP4 need no LDS (64 sequences of 8192 tokens, 8 heads: 115.6 -> 109.0 us).  Those of a + format do better by it: the block
  // maximum costs 30 vector instructions in registers and one store there (4 % slower in registers).
  constexpr bool KEYS_IN_REGISTERS = D >= 128 && MODE == 0;
  constexpr int DB = D / 32, NB = D / 64, PATCH = few_patch<D>(NT);   // blocks per token; per lane of a 32-token tile
  constexpr int LANE_TOKENS = D == 64 ? 32 : 16;             // tokens that a wavefront's lanes cover with one block each (of 2, 4, 4 neighbours)
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  uint8_t* const patch = lds + wave * PATCH;                 // a tile's keys, then its values
  float* const ml = reinterpret_cast<float*>(lds + WAVES * PATCH);   // [wave][row][2]
  // This lane's blocks of a tile: the first one's token (16 lanes in a row have 16 tokens: their stores fall on all banks) and its block
  // of the token; how far on the i-th is
  const int lane_token = lane & (LANE_TOKENS - 1), lane_block = lane / LANE_TOKENS;
  const auto tokens_on = [](int i) { return D == 256 ? 16 * (i >> 1) : LANE_TOKENS * i; };
  const auto blocks_on = [](int i) { return D == 256 ? 4 * (i & 1) : 0; };
  constexpr int ROWS = 16 * NT;
  __shared__ Share share;
  __shared__ int64_t wave_sum[kWaves];
  for (Walk<DIRECT> walk(a, ROWS, kFewUnit, kFewLeast, false, share, wave_sum);;) {
    if (!walk.more(a)) break;
    const Sequence s(a, walk.seq);
    if (!walk.more(a, s, ROWS)) break;
    int r0 = 0;
    Span span;
    if (!walk.next(a, s, ROWS, kFewUnit, share, r0, span)) continue;
    const int R = s.n * a.group, kv_head = walk.kv_head, part = walk.part;
    // this lane's rows, as operands of the first product: eight channels per step
    Operand q[NT][DB];
    int first[NT];                                           // what a row sees of the span: from here,
    uint32_t seen[NT];                                       // so many tokens
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = r0 + 16 * t + col, i = r / a.group;
      const bool there = r < R;
      first[t] = s.first(a, i);
      seen[t] = there ? tokens_from_to(first[t], s.last(a, i), span.end) : 0u;
      const uint16_t* p = a.q + (s.q0 + (there ? i : 0)) * a.ld_q + (int64_t)(kv_head * a.group + (there ? r - i * a.group : 0)) * D + (KEYS_IN_REGISTERS ? 32 : 8) * quarter;
#pragma unroll
      for (int st = 0; st < DB; ++st) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + (KEYS_IN_REGISTERS ? 128 * (st >> 2) + 8 * (st & 3) : 32 * st));
#pragma unroll
        for (int j = 0; j < 4; ++j) q[t][st].u[j] = there ? x[j] ^ a.flip : 0u;
      }
    }
    // tokens that every row of the tile sees
    const int all_from = s.first(a, (R - r0 < 16 * NT ? R - 1 : r0 + 16 * NT - 1) / a.group), all_to = s.last(a, r0 / a.group);
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t] = -kInf;
      l[t] = 0.0f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[t][d] = f32x4{0, 0, 0, 0};
    }
    // The wavefront's tiles: span.begin + 32 wave, and every 32 WAVES tokens from there.  Lane n holds the page of half n % 2 of
    // tile n / 2 of the next 32 tiles (-1: none), so that a tile's addresses wait for no table.
    const int begin = span.begin + 32 * wave;
    int fetched = 0;                                         // tiles
    int32_t pages = -1;
    struct Fetched {                                         // a tile's blocks on their way, and whether its halves have a page
      Block k[NB], v[NB];
      bool held0, held1;
    } ahead[kFewAhead];
    const auto fetch = [&](Fetched& f, int t) {
      if (t >= span.end) return;
      if ((fetched & 31) == 0) pages = page_of(a, s, (int64_t)t + 32 * WAVES * (lane >> 1) + 16 * (lane & 1));
      const Page p0(a, kv_head, __builtin_amdgcn_readlane(pages, 2 * (fetched & 31)), t), p1(a, kv_head, __builtin_amdgcn_readlane(pages, 2 * (fetched & 31) + 1), t + 16);
      f.held0 = p0.held;
      f.held1 = p1.held;
      ++fetched;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const bool second = D == 64 ? lane_token >= 16 : tokens_on(i) >= 16;
        const uint8_t* rec = second ? p1.rec : p0.rec;
        const int row = (second ? p1.at : p0.at) + (lane_token & 15);
        f.k[i] = load_block<D, MODE, true>(rec, a.g, row, lane_block + blocks_on(i));
        f.v[i] = load_block<D, MODE, true>(rec + a.g.part_bytes, a.g, row, lane_block + blocks_on(i));
      }
    };
    const uint32_t lane_at = token_at<D>(lane_token) ^ (64u * lane_block);
    const auto take = [&](Fetched& f, int t0) {
      if (t0 >= span.end) return;
      const bool h0 = f.held0, h1 = f.held1;
      uint64_t nan[NB];                                      // lanes whose block of V is NaN: zeros here, put in behind the product
      uint64_t any = 0;
      f32x4 sc[NT][2];
      if constexpr (KEYS_IN_REGISTERS) {
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          Operand k[4];
          expand(f.k[i], k);
          const int h = tokens_on(i) >> 4;
#pragma unroll
          for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int t = 0; t < NT; ++t) sc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[st].v, q[t][blocks_on(i) + st].v, sc[t][h], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NB; ++i) expand<MODE>(f.k[i], false, patch + 2 * D * tokens_on(i), formed_at_use(lane_at) ^ (64u * blocks_on(i)));
        __builtin_amdgcn_wave_barrier();
        const uint32_t k_at = formed_at_use(token_at<D>(col) ^ (16u * quarter));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][h] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int st = 0; st < DB; ++st) {
            Operand k;
            const u32x4 x = *reinterpret_cast<const u32x4*>(patch + 32 * D * h + (k_at ^ (64u * st)));
#pragma unroll
            for (int j = 0; j < 4; ++j) k.u[j] = x[j];
#pragma unroll
            for (int t = 0; t < NT; ++t) sc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v, q[t][st].v, sc[t][h], 0, 0, 0);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();                       // (the reads above come first: LDS serves a wavefront in order)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int token = lane_token + tokens_on(i);
        const bool dead = t0 + token >= span.end || !(token >= 16 ? h1 : h0);
        nan[i] = __ballot(f.v[i].scale == 255u && !dead);
        any |= nan[i];
        expand<MODE>(f.v[i], dead || f.v[i].scale == 255u, patch + 2 * D * tokens_on(i), formed_at_use(lane_at) ^ (64u * blocks_on(i)));
      }
      __builtin_amdgcn_wave_barrier();
      fetch(f, t0 + kFewAhead * 32 * WAVES);
      const bool whole = h0 && h1 && t0 >= all_from && t0 + 31 <= all_to && t0 + 32 <= span.end;   // (uniform)
      if (!whole) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t from_first = (uint32_t)(t0 + 4 * quarter - first[t]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[t][h][i] = from_first + 16u * h + i < seen[t] && (h ? h1 : h0) ? sc[t][h][i] : -kInf;
        }
      }
      Operand p[NT][TERMS];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float mx = fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), fmaxf(sc[t][0][2], sc[t][0][3])), fmaxf(fmaxf(sc[t][1][0], sc[t][1][1]), fmaxf(sc[t][1][2], sc[t][1][3])));
        mx = fmaxf(m[t], max_across_32(max_across_16(mx)));
        if (__any(mx > m[t])) {
          mx = raised(m[t], mx, a.up);
          const float fade = exp2_of((m[t] - zero_if_none(mx)) * a.scale);
          l[t] *= fade;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) o[t][d] *= fade;
          m[t] = mx;
        }
        const float base = zero_if_none(m[t]) * a.scale;
        l[t] += weights<TERMS>(sc[t][0], sc[t][1], a.scale, base, p[t]);
      }
      const uint32_t v_at = formed_at_use(token_at<D>(4 * quarter + (col >> 2)) ^ (8u * (col & 3)));
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        Operand v;
        const uint8_t* at = patch + (v_at ^ (32u * d));
        v.s[0] = read_transposed(at);
        v.s[1] = read_transposed(at + 32 * D);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int c = 0; c < TERMS; ++c) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, p[t][c].v, o[t][d], 0, 0, 0);
      }
      if (any) {                                             // NaN blocks of V, for the rows that see them
#pragma unroll 1
        for (int i = 0; i < NB; ++i) {
          uint64_t left = nan[0];
#pragma unroll
          for (int k = 1; k < NB; ++k) left = i == k ? nan[k] : left;
          for (; left; left &= left - 1) {
            const int who = __builtin_ctzll(left), tok = t0 + (who & (LANE_TOKENS - 1)) + tokens_on(i), blk = who / LANE_TOKENS + blocks_on(i);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const bool sees = (uint32_t)(tok - first[t]) < seen[t];
#pragma unroll
              for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[t][d][j] = sees && d / 2 == blk ? __uint_as_float(0x7FC00000u) : o[t][d][j];
            }
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) fetch(ahead[u], begin + u * 32 * WAVES);
    if (begin < span.first && begin < span.end) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (begin + lane_token + tokens_on(i) < span.first) ahead[0].v[i].blank();
    }
    for (int t0 = begin; t0 < span.end; t0 += kFewAhead * 32 * WAVES)
#pragma unroll
      for (int u = 0; u < kFewAhead; ++u) take(ahead[u], t0 + u * 32 * WAVES);
    // join the wavefronts: each leaves its rows in its own patch
    float* const mine = reinterpret_cast<float*>(patch);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float sum = sum_across_32(sum_across_16(l[t]));
      if (quarter == 0) {
        ml[(wave * 16 * NT + 16 * t + col) * 2] = m[t] * a.scale;
        ml[(wave * 16 * NT + 16 * t + col) * 2 + 1] = sum;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(mine + (16 * t + col) * D + 16 * d + 4 * quarter) = o[t][d];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 16 * NT * (D / 4); j += 64 * WAVES) {
      const int row = j / (D / 4), d = (j - row * (D / 4)) * 4, r = r0 + row;
      if (r >= R) break;
      float top = -kInf, sum = 0.0f;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) top = fmaxf(top, ml[(v * 16 * NT + row) * 2]);
      const float base = zero_if_none(top);
      f32x4 out = {0, 0, 0, 0};
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const float f = exp2_of(ml[(v * 16 * NT + row) * 2] - base);
        sum += ml[(v * 16 * NT + row) * 2 + 1] * f;
        out += *reinterpret_cast<const f32x4*>(lds + v * PATCH + (row * D + d) * 4) * f;
      }
      const int i = r / a.group, head = kv_head * a.group + r - i * a.group;
      const int64_t part_row = part < 0 ? -1 : (int64_t)part * ROWS + row;
      finish_values(a, part_row, s.q0 + i, head, d, out, sum);
      if (d == 0) finish_row(a, part_row, s.q0 + i, head, top, sum);
    }
    __syncthreads();
  }
}

// Four values of a row per lane, for at most P parts: every lane forms the weights by itself.  (The places behind the last part load the
// first one again: loads under a condition each are not under way together, and the chunks below then take 155 us instead of 148.)
template <int P>
struct FewParts {
  float m[P], l[P];
  f32x4 x[P];
  template <class PartAt>
  __device__ __forceinline__ void load(const AttnArgs& a, int parts, PartAt part_at, int d) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t at = part_at(p < parts ? p : 0);
      m[p] = p < parts ? a.part_ml[2 * at] : -kInf;
      l[p] = p < parts ? a.part_ml[2 * at + 1] : 0.0f;
      x[p] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.part_o + at * a.g.D + d));
    }
  }
  __device__ __forceinline__ void finish(const AttnArgs& a, int64_t row, int head, int d) const {
    float top = -kInf, sum = 0.0f;
    f32x4 out = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < P; ++p) top = fmaxf(top, m[p]);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if (l[p] == 0.0f) continue;
      const float f = exp2_of(m[p] - zero_if_none(top));
      sum += l[p] * f;
      out += x[p] * f;
    }
    store_out(a, row, head, d, sum == 0.0f ? f32x4{0, 0, 0, 0} : out / sum);
    if (d == 0 && a.lse) a.lse[row * a.heads + head] = lse_of(top, sum);
  }
};

// A tile of rows from at most P parts: a lane's four values of ROWS rows, their loads under way together.  (Three chunks of 777
// queries behind 3000 to 9001 tokens, 294 tiles of 128 rows in 512 shares: 24 us with one row at once and 16 rows per workgroup, 14.7
// with two and 64; two and 32: 17.2, four and 64: 19.2.  Eleven of up to 559 queries, with five to eight parts where a wavefront took
// a row before: 83 -> 78 us in all.)
template <int P, int ROWS>
__device__ __forceinline__ void join_tile(const AttnArgs& a, const Sequence& s, int kv_head, int r0, int rows, int rows_per_tile, int first, int parts) {
  const int shift = __builtin_ctz(a.g.D >> 2), d = 4 * ((int)threadIdx.x & ((a.g.D >> 2) - 1)), step = (256 >> shift) * (int)gridDim.y;
  for (int row = (int)blockIdx.y * (256 >> shift) + ((int)threadIdx.x >> shift); row < rows; row += ROWS * step) {
    FewParts<P> f[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
      if (row + u * step < rows) f[u].load(a, parts, [&](int p) { return ((int64_t)2 * (first + p) + (p == 0 ? 1 : 0)) * rows_per_tile + row + u * step; }, d);
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const int r = r0 + row + u * step, query = r / a.group;
      if (row + u * step < rows) f[u].finish(a, s.q0 + query, kv_head * a.group + r - query * a.group, d);
    }
  }
}

// The joins that Share records, `each` workgroups' records per workgroup here, in the way that fits the parts: few, up to 64, more.
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnArgs a, int rows_per_tile, int n_records, int each) {
  __shared__ JoinRoom room;
  const int lane = threadIdx.x & 63, first = (int)blockIdx.x * each;
  uint64_t todo = __ballot(lane < each && first + lane < n_records && a.joins[4 * (first + lane)] >= 0);
  for (; todo; todo &= todo - 1) {                           // (the same in every wavefront)
    const int g = first + __builtin_ctzll(todo);
    const int32_t* const j = a.joins + 4 * g;
    const Sequence s(a, j[0]);
    const int kv_head = j[1], r0 = j[2], parts = j[3] - g + 1, R = s.n * a.group;
    if (parts <= 8) {
      const int rows = R - r0 < rows_per_tile ? R - r0 : rows_per_tile;
      if (parts <= 4) join_tile<4, 2>(a, s, kv_head, r0, rows, rows_per_tile, g, parts);
      else join_tile<8, 1>(a, s, kv_head, r0, rows, rows_per_tile, g, parts);
      continue;
    }
    const bool by_wave = parts <= 64;
    const int step = (by_wave ? 4 : 1) * (int)gridDim.y;
    for (int row = by_wave ? (int)blockIdx.y * 4 + (int)(threadIdx.x >> 6) : (int)blockIdx.y; row < rows_per_tile && r0 + row < R; row += step) {
      const int r = r0 + row, i = r / a.group;
      const auto part_at = [&](int p) { return ((int64_t)2 * (g + p) + (p == 0 ? 1 : 0)) * rows_per_tile + row; };
      if (by_wave) join_row_by_wave(a, parts, part_at, s.q0 + i, kv_head * a.group + r - i * a.group);
      else join_row(a, room, parts, part_at, s.q0 + i, kv_head * a.group + r - i * a.group);
    }
  }
}

// ---- many rows ------------------------------------------------------------------------------------------------------
constexpr int kManyTokens = 64, kManyRows = 32 * kWaves, kManyLeast = 8;   // (a unit is a tile of tokens)
template <int D>
constexpr int many_jobs() { return 2 * kManyTokens * (D / 32) / (64 * kWaves); }   // blocks of a tile per lane
template <int D>
constexpr int many_lds() { return 2 * 2 * kManyTokens * 2 * D + 2 * kWaves * many_jobs<D>() * 8; }   // two buffers of keys and values; NaN masks

template <int D, int MODE, int TERMS, bool DIRECT>
__global__ void __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) attn_many_kernel(const AttnArgs a) {
  constexpr int DB = D / 32, HALF = kManyTokens * 2 * D, JOBS = many_jobs<D>();
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  uint64_t* const nans = reinterpret_cast<uint64_t*>(lds + 4 * HALF);   // [buffer][wave][job] lanes with a NaN block of V
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  // The blocks of a tile that wavefront w expands, D >= 128: tokens 16 w ... + 15, keys in even jobs, values in odd ones, four blocks of a
  // token per job; D = 64: tokens 32 (w % 2) ... + 31, keys for w < 2, values for the others
  const auto job_of_v = [&](int k) { return D == 64 ? wave >> 1 : k & 1; };
  const auto job_token = [&](int w, int who) { return D == 64 ? 32 * (w & 1) + (who & 31) : 16 * w + (who & 15); };
  const auto job_block = [&](int k, int who) { return D == 64 ? who >> 5 : 4 * (k >> 1) + (who >> 4); };
  __shared__ Share share;
  __shared__ int64_t wave_sum[kWaves];
  for (Walk<DIRECT> walk(a, kManyRows, kManyTokens, kManyLeast, true, share, wave_sum);;) {
    if (!walk.more(a)) break;
    const Sequence s(a, walk.seq);
    if (!walk.more(a, s, kManyRows)) break;
    int r0 = 0;
    Span span;
    if (!walk.next(a, s, kManyRows, kManyTokens, share, r0, span)) continue;
    const int R = s.n * a.group, kv_head = walk.kv_head, part = walk.part;
    const int r = r0 + 32 * wave + col, i = r / a.group;
    const bool there = r < R;
    const int first = s.first(a, i);                         // what the row sees of the span: from here,
    const uint32_t seen = there ? tokens_from_to(first, s.last(a, i), span.end) : 0u;   // so many tokens
    const int head = kv_head * a.group + (there ? r - i * a.group : 0);
    Operand q[D / 16];
    {
      const uint16_t* p = a.q + (s.q0 + (there ? i : 0)) * a.ld_q + (int64_t)head * D + 8 * half;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + 16 * st);
#pragma unroll
        for (int j = 0; j < 4; ++j) q[st].u[j] = there ? x[j] ^ a.flip : 0u;
      }
    }
    // what the wavefront's rows see: some of them, all of them
    const int wr0 = r0 + 32 * wave, wr1 = (wr0 + 31 < R ? wr0 + 31 : R - 1);
    const bool rows_here = wr0 < R;
    const int any_from = rows_here ? s.first(a, wr0 / a.group) : 0, any_to = rows_here ? s.last(a, wr1 / a.group) : -1;
    const int all_from = rows_here ? s.first(a, wr1 / a.group) : 0, all_to = rows_here ? s.last(a, wr0 / a.group) : -1;
    f32x16 o[DB];
    float m = -kInf, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[d][j] = 0.0f;
    Block job[JOBS];
    uint32_t held = 0, held_next = 0;                        // bit j: tokens 16 j ... + 15 of the tile have a page
    int fetched = 0;                                         // tiles
    int32_t pages = -1;                                      // lane n: the page of tokens 16 (n % 4) ... of tile n / 4 of the next 16
    const auto fetch = [&](int t) {
      if ((fetched & 15) == 0) pages = page_of(a, s, (int64_t)t + 16 * lane);
      held_next = 0;
      int32_t number[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        number[j] = __builtin_amdgcn_readlane(pages, 4 * (fetched & 15) + j);
        held_next |= (number[j] >= 0 ? 1u : 0u) << j;
      }
      ++fetched;
      // this wavefront's tokens lie in one 16-token group of the tile (D = 64: in two)
      const int group = D == 64 ? 2 * (wave & 1) : wave;
      const int32_t n0 = D == 64 ? (wave & 1 ? number[2] : number[0]) : wave & 2 ? (wave & 1 ? number[3] : number[2]) : (wave & 1 ? number[1] : number[0]);
      const Page p0(a, kv_head, n0, t + 16 * group), p1(a, kv_head, D == 64 ? (wave & 1 ? number[3] : number[1]) : n0, t + 16 * group + 16);
      const bool second = D == 64 && (lane & 16);
      const uint8_t* const rec = second ? p1.rec : p0.rec;
      const int row = (second ? p1.at : p0.at) + (lane & 15);
#pragma unroll
      for (int k = 0; k < JOBS; ++k) job[k] = load_block<D, MODE, false>(rec + (job_of_v(k) ? a.g.part_bytes : 0), a.g, row, job_block(k, lane));
    };
    const auto expand_all = [&](int t, int buf) {            // the fetched tile into a buffer
      const int token = job_token(wave, lane);
      const bool dead = t + token >= span.end || !((held_next >> (token >> 4)) & 1u);
#pragma unroll
      for (int k = 0; k < JOBS; ++k) {
        const bool nan = job_of_v(k) && job[k].scale == 255u;
        expand<MODE>(job[k], job_of_v(k) && (dead || nan), lds + buf * 2 * HALF + job_of_v(k) * HALF, token_at<D>(token) ^ (64u * job_block(k, lane)));
        const uint64_t b = __ballot(nan && !dead);
        if (lane == 0) nans[(buf * kWaves + wave) * JOBS + k] = b;
      }
    };
    int buf = 0;
    if (span.begin < span.end) {
      fetch(span.begin);
      if (span.begin < span.first) {
#pragma unroll
        for (int k = 0; k < JOBS; ++k)
          if (job_of_v(k) && span.begin + job_token(wave, lane) < span.first) job[k].blank();
      }
      expand_all(span.begin, 0);
    }
    for (int t0 = span.begin; t0 < span.end; t0 += kManyTokens) {
      held = held_next;
      const bool more = t0 + kManyTokens < span.end;
      __syncthreads();                                       // the tile is there
      if (more) fetch(t0 + kManyTokens);
      const uint8_t* const kt = lds + buf * 2 * HALF;
      const uint8_t* const vt = kt + HALF;
      if (t0 <= any_to && t0 + kManyTokens > any_from) {     // (uniform in the wavefront)
        f32x16 sc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int j = 0; j < 16; ++j) sc[h][j] = 0.0f;
#pragma unroll
          for (int st = 0; st < D / 16; ++st) {
            Operand k;
            const u32x4 x = *reinterpret_cast<const u32x4*>(kt + 64 * D * h + (token_at<D>(col) ^ (16u * half) ^ (32u * st)));
#pragma unroll
            for (int j = 0; j < 4; ++j) k.u[j] = x[j];
            sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.v, q[st].v, sc[h], 0, 0, 0);
          }
        }
        const bool whole = held == 15u && t0 >= all_from && t0 + kManyTokens - 1 <= all_to && t0 + kManyTokens <= span.end;
        if (!whole) {
          const uint32_t from_first = (uint32_t)(t0 + 4 * half - first);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 16; ++j) sc[h][j] = from_first + (32u * h + 8 * (j >> 2) + (j & 3)) < seen ? sc[h][j] : -kInf;
          if (held != 15u) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int j = 0; j < 16; ++j) sc[h][j] = (held >> (2 * h + (j >> 3))) & 1u ? sc[h][j] : -kInf;
          }
        }
        float mx = -kInf;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 16; ++j) mx = fmaxf(mx, sc[h][j]);
        mx = fmaxf(m, max_across_32(mx));
        if (__any(mx > m)) {
          mx = raised(m, mx, a.up);
          const float fade = exp2_of((m - zero_if_none(mx)) * a.scale);
          l *= fade;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d] *= fade;
          m = mx;
        }
        const float base = zero_if_none(m) * a.scale;
#pragma unroll
        for (int b = 0; b < 4; ++b) {                        // 16 tokens: registers 8 (b % 2) ... + 7 of half b / 2
          Operand p[TERMS];
          const int j = 8 * (b & 1);
          const f32x16& x = sc[b >> 1];
          l += weights<TERMS>(f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]}, f32x4{x[j + 4], x[j + 5], x[j + 6], x[j + 7]}, a.scale, base, p);
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            Operand v;
            const uint32_t at = token_at<D>(4 * half + ((lane & 15) >> 2)) ^ (32u * ((lane >> 4) & 1)) ^ (8u * (lane & 3)) ^ (64u * d);
            v.s[0] = read_transposed(vt + 32 * D * b + at);
            v.s[1] = read_transposed(vt + 32 * D * b + 16 * D + (at ^ 32u));   // eight tokens on: s differs in bit 1
#pragma unroll
            for (int c = 0; c < TERMS; ++c) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, p[c].v, o[d], 0, 0, 0);
          }
        }
        uint64_t any = 0;
#pragma unroll
        for (int k = 0; k < kWaves * JOBS; ++k) any |= nans[buf * kWaves * JOBS + k];
        if (__any(any != 0)) {                               // NaN blocks of V, for the rows that see them
#pragma unroll 1
          for (int k = 0; k < kWaves * JOBS; ++k)
            for (uint64_t left = nans[buf * kWaves * JOBS + k]; left; left &= left - 1) {
              const int who = __builtin_ctzll(left), tok = t0 + job_token(k / JOBS, who), blk = job_block(k % JOBS, who);
              const bool sees = (uint32_t)(tok - first) < seen;
#pragma unroll
              for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[d][j] = sees && d == blk ? __uint_as_float(0x7FC00000u) : o[d][j];
            }
        }
      }
      if (more) {
        buf ^= 1;
        expand_all(t0 + kManyTokens, buf);
      }
    }
    l = sum_across_32(l);
    if (m * a.scale == kInf) l = __builtin_nanf("");         // (scores beyond fp32, all weights 0: not a row that sees nothing)
    if (there) {
      const int64_t part_row = part < 0 ? -1 : (int64_t)part * kManyRows + 32 * wave + col;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          finish_values(a, part_row, s.q0 + i, head, 32 * d + 8 * j + 4 * half, f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]}, l);
      if (half == 0) finish_row(a, part_row, s.q0 + i, head, m * a.scale, l);
    }
    __syncthreads();
  }
}

// ---- launch -----------------------------------------------------------------------------------------------------------
struct Plan {
  bool many, direct, alone;                                  // alone: a workgroup per compute unit at most
  int rows, row_tiles;                                       // of a tile, tiles per key-value head and sequence
  int64_t wgs;
};

// Sequences of at most so many tokens are not dealt out in parts: a workgroup goes over them in less than the parts' join takes.
// (Few rows, us whole | dealt out, tiles of rows of 1024 tokens, of 2048, head_dim 128: 8 tiles 14.3 | 14.0, 22.2 | 15.1; 32: 15.0 | 14.6,
// 22.4 | 15.5; 64: 15.4 | 14.8, 22.8 | 18.2; 80: 15.6 | 20.0, 22.9 | 21.6; 128: 15.7 | 18.1, 23.2 | 22.3; 320: 23.6 | 26.2, 38.5 | 41.5;
// MXFP4++ the same within 0.4 us, of 1024 tokens at 8 tiles 15.5 | 14.7.  At head_dim 256 whole tiles are behind at more tiles too:
// 8: 25.9 | 19.4, 38.8 | 20.2; 64: 26.6 | 20.3, 41.7 | 26.6; 80: 26.8 | 28.2, 41.8 | 33.0; 128: 27.2 | 26.4, 42.4 | 34.7; 320: 43.1 | 44.9,
// 71.5 | 65.1; the rule does not heed it.)
constexpr int64_t kFewDirect = 2048, kFewestDirect = 512, kManyDirect = 1024;

// Which kernel (up to 32 rows of a key-value head: attn_few_kernel), and whether a workgroup takes whole tiles of rows or a share of
// all tokens.  Whole tiles where sequences are short, where workgroups come in several rounds anyhow (they then even out among
// themselves), and for prompts: a tile of theirs sees half the tokens on average, which shares of equal numbers of tokens do not heed.
// Shares where the bound on a sequence's queries is far above what most have (a prompt among single queries): whole tiles would
// be mostly empty workgroups.
Plan plan_for(int64_t n_seq, int64_t rows, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads, int64_t D, int causal, int64_t window) {
  Plan p;
  max_q = max_q < rows ? max_q : rows;
  window = window < kMostTokens ? window : kMostTokens;
  const int64_t group = heads / kv_heads, most = max_q * group;
  p.many = most > 32;
  p.rows = p.many ? kManyRows : most > 16 ? 32 : 16;
  p.row_tiles = (int)((most + p.rows - 1) / p.rows);
  if (p.row_tiles < 1) p.row_tiles = 1;
  const int64_t items = n_seq * kv_heads * p.row_tiles, filled = kv_heads * ((rows * group + p.rows - 1) / p.rows + n_seq), real = items < filled ? items : filled;
  int64_t len = max_kv;                                      // tokens that one tile of rows goes over, at most
  if (window > 0 && window + max_q + 32 < len) len = window + max_q + 32;
  const int64_t room = (int64_t)kNumCU * (p.many ? (D == 256 ? 1 : 2) : few_waves_per_simd((int)D, p.rows / 16));   // workgroups that run at once
  const int64_t unit = p.many ? kManyTokens : kFewUnit, least = p.many ? kManyLeast : kFewLeast;
  const int64_t shares = shares_of(real * ((len + unit - 1) / unit), least);
  const bool prompt = p.many && causal && 2 * max_q > len && 2 * items > room;
  p.direct = items <= 2 * real + room && (len <= (p.many ? kManyDirect : items > 64 ? kFewDirect : kFewestDirect) || items >= 4 * room || prompt);
  p.alone = !p.many && p.direct && items <= kNumCU;
  p.wgs = p.direct ? items : shares < 1 ? 1 : shares < room ? shares : room;
  return p;
}

// Workspace: values of the parts, their maxima and sums, records of joins
int64_t part_rows(const Plan& p) { return p.direct ? 0 : p.wgs * 2 * p.rows; }
size_t parts_bytes(const Plan& p, int64_t D) { return p.direct ? 0 : (size_t)part_rows(p) * (size_t)(D + 2) * 4 + (size_t)p.wgs * 16; }

template <int D, int MODE, int NT, int TERMS, int WAVES, bool DIRECT>
void launch_few(const AttnArgs& a, const Plan& p, hipStream_t s) {
  constexpr int bytes = few_lds<D>(NT, WAVES);
  allow_dynamic_lds<attn_few_kernel<D, MODE, NT, TERMS, WAVES, DIRECT>>(bytes);
  hipLaunchKernelGGL((attn_few_kernel<D, MODE, NT, TERMS, WAVES, DIRECT>), dim3((unsigned)p.wgs), dim3(64 * WAVES), bytes, s, a);
}
template <int D, int MODE, int NT, int TERMS>
void launch_few(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.alone) launch_few<D, MODE, NT, TERMS, few_waves_alone(D, NT), true>(a, p, s);
  else if (p.direct) launch_few<D, MODE, NT, TERMS, kWaves, true>(a, p, s);
  else launch_few<D, MODE, NT, TERMS, kWaves, false>(a, p, s);
}

template <int D, int MODE, int TERMS, bool DIRECT>
void launch_many(const AttnArgs& a, const Plan& p, hipStream_t s) {
  allow_dynamic_lds<attn_many_kernel<D, MODE, TERMS, DIRECT>>(many_lds<D>());
  hipLaunchKernelGGL((attn_many_kernel<D, MODE, TERMS, DIRECT>), dim3((unsigned)p.wgs), dim3(64 * kWaves), many_lds<D>(), s, a);
}

template <int D, int MODE, int TERMS>
void launch(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.many) {
    if (p.direct) launch_many<D, MODE, TERMS, true>(a, p, s);
    else launch_many<D, MODE, TERMS, false>(a, p, s);
  } else if (p.rows == 32) {
    launch_few<D, MODE, 2, TERMS>(a, p, s);
  } else {
    launch_few<D, MODE, 1, TERMS>(a, p, s);
  }
}

// shape rules that the size function and the call share
bool shapes_fit(int64_t n_seq, int64_t rows, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads) {
  return n_seq >= 0 && rows >= 0 && max_q >= 0 && max_kv >= 0 && heads >= 1 && heads <= 65535 && kv_heads >= 1 && heads % kv_heads == 0 &&
         rows <= 2147483647LL && max_q <= 2147483647LL && max_kv <= 2147483647LL && n_seq <= 2147483647LL;
}

}  // namespace

extern "C" size_t mxp_attention_workspace_bytes(int64_t n_seq, int64_t rows, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads,
                                                int64_t head_dim, int causal, int64_t window) {
  if (!shapes_fit(n_seq, rows, max_q, max_kv, heads, kv_heads) || n_seq == 0 || rows == 0 || rows * heads > kMostRows || head_dim < 1 || window < 0) return 0;
  return parts_bytes(plan_for(n_seq, rows, max_q, max_kv, heads, kv_heads, head_dim, causal, window), head_dim);
}

extern "C" int mxp_attention(const void* Q, int q_dtype, int64_t ld_q, int64_t rows, int64_t heads, const int32_t* q_start, const int32_t* kv_len,
                             const int32_t* table, int64_t ld_table, int64_t n_seq, int64_t max_q, int64_t max_kv, float scale, int causal,
                             int64_t window, const void* cache, int64_t n_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim, int fmt,
                             void* O, int o_dtype, int64_t ld_o, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace mxp;
  AttnArgs a;
  const int rc = cache_geom(n_pages, page_tokens, kv_heads, head_dim, fmt, a.g);
  if (rc != MXP_OK) return rc;
  if ((q_dtype != MXP_F32 && q_dtype != MXP_BF16) || (o_dtype != MXP_F32 && o_dtype != MXP_BF16)) return MXP_ERR_DTYPE;
  if (!shapes_fit(n_seq, rows, max_q, max_kv, heads, kv_heads) || ld_table < 0 || window < 0 || (window > 0 && !causal) ||
      !(scale > -__builtin_inff() && scale < __builtin_inff()) || (!q_start && rows != n_seq))
    return MXP_ERR_SHAPE;
  if (q_dtype == MXP_F32 || rows * heads > kMostRows) return MXP_ERR_UNSUPPORTED;
  if (rows == 0 || n_seq == 0) return MXP_OK;
  if (!Q || !kv_len || !O || !cache || (ld_table > 0 && !table)) return MXP_ERR_NULL;
  const int64_t width = heads * head_dim, osz = o_dtype == MXP_BF16 ? 2 : 4;
  if (ld_q < width || ld_o < width) return MXP_ERR_SHAPE;
  const auto off4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; };
  if (!aligned16(Q) || !aligned16(O) || !aligned16(cache) || !aligned16(workspace) || ld_q * 2 % 16 != 0 || ld_o * osz % 16 != 0 || off4(q_start) ||
      off4(kv_len) || off4(table) || off4(lse))
    return MXP_ERR_ALIGN;
  const Plan p = plan_for(n_seq, rows, max_q, max_kv, heads, kv_heads, head_dim, causal, window);
  if (p.wgs >= ((int64_t)1 << 24)) return MXP_ERR_UNSUPPORTED;   // (a launch has fewer than 2^32 threads)
  const size_t need = parts_bytes(p, head_dim);
  if (need > 0 && (!workspace || workspace_bytes < need)) return MXP_ERR_WORKSPACE;
  a.q = static_cast<const uint16_t*>(Q);
  a.ld_q = ld_q;
  a.rows = rows;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.table = table;
  a.ld_table = ld_table;
  a.n_seq = (int)n_seq;
  a.heads = (int)heads;
  a.group = (int)(heads / kv_heads);
  a.causal = causal ? 1 : 0;
  a.window = (int)(window < 2147483647LL ? window : 2147483647LL);
  a.scale = (scale < 0 ? -scale : scale) * 1.4426950408889634f;
  if (a.scale < 1.17549435e-38f) a.scale = 1.17549435e-38f;   // (0 would make NaN of a hidden token's -infinity,
  if (a.scale > kMostFloat) a.scale = kMostFloat;             // infinity of a score of 0)
  a.up = kGrowth / a.scale < 8.5e37f ? kGrowth / a.scale : 8.5e37f;   // (a number: -infinity stays where nothing was seen)
  a.flip = scale < 0 ? 0x80008000u : 0u;
  a.data = static_cast<const uint8_t*>(cache);
  a.o = O;
  a.ld_o = ld_o;
  a.o_bf16 = o_dtype == MXP_BF16;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  const size_t parts = (size_t)part_rows(p);
  a.part_ml = need ? a.part_o + parts * head_dim : nullptr;
  a.joins = need ? reinterpret_cast<int32_t*>(a.part_ml + 2 * parts) : nullptr;
  a.row_tiles = p.row_tiles;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_ATTN_T(D, M) do { if (a.o_bf16) launch<D, M, 1>(a, p, s); else launch<D, M, 3>(a, p, s); } while (0)
#define MXP_ATTN_M(D) do { if (fmt == MXP_FMT_MXFP4) MXP_ATTN_T(D, 0); else if (fmt == MXP_FMT_MXFP4P) MXP_ATTN_T(D, 1); else MXP_ATTN_T(D, 2); } while (0)
  if (head_dim == 64) MXP_ATTN_M(64);
  else if (head_dim == 128) MXP_ATTN_M(128);
  else MXP_ATTN_M(256);
#undef MXP_ATTN_M
#undef MXP_ATTN_T
  if (!p.direct) {
    // About so many parts a join: above 32 there are few records, 16 of them and one row per workgroup (one sequence of 131000 tokens,
    // 8 joins of 128 parts: 14.6 -> 7.8 us against a record each); else a record per workgroup, one row per wavefront or, where
    // joins have about as few parts as join_tile takes (twice the average in the longest sequences), 64 rows.
    const int64_t parts_each = p.wgs / (n_seq * kv_heads * p.row_tiles);
    int64_t most = (max_q < rows ? max_q : rows) * a.group;
    most = most < 1 ? 1 : most < p.rows ? most : p.rows;
    const int each = parts_each >= 32 ? 16 : 1;
    const int64_t y = parts_each >= 32 ? most : parts_each >= 4 ? (most + 3) / 4 : (most + 63) / 64;
    hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)((p.wgs + each - 1) / each), (unsigned)y), dim3(256), 0, s, a, p.rows,
                       (int)p.wgs, each);
  }
  return launch_status();
}
