// mxp_attention: softmax attention of ragged query rows over the paged four-bit cache (layout: mxp_cache.h).
//
// One pass over the visible tokens with the running maximum and sum of the softmax, in base 2 (the scale carries log2 e):
//     S = K Q^T     m' = max(m, S)     P = 2^(S - m')     l = l 2^(m - m') + sum P     O = O 2^(m - m') + V^T P
// Both products have the tokens' side as their first operand, so the result of the first, [token][row], has a query row per lane
// column and four or sixteen tokens in a lane's registers: what the second takes as its second operand, up to a permutation of the
// tokens inside one MFMA step, which the reads of V follow.  Maximum, sum and rescaling are then a lane's own business (plus one
// exchange between the lanes of a column), and P never leaves the registers.
//
// Keys and values are de-converted (Eq. 2, exact in bf16) into LDS, a lane per block: 16 unpack-converts, four 16-byte stores, and
// the block maximum of a + format as one 2-byte store over its element, which costs a fifth of merging it in registers.  V is read
// back transposed by the LDS hardware (4 tokens x 16 channels per 16 lanes).
//
// Query rows of one key-value head (heads that share it x queries) are taken together.  attn_few_kernel: up to 32 of them per
// workgroup, every wavefront with tokens of its own, joined through LDS at the end; bound by reading the cache.
// attn_many_kernel: 128 rows per workgroup, the wavefronts share the de-converted tokens; bound by the matrix cores and the softmax.
// Both can split a sequence's tokens over workgroups; attn_join_kernel then adds the parts.
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
  float scale;                                               // |scale| * log2(e), at least the smallest normal number
  uint32_t flip;                                             // sign bits of two bf16 where scale is negative: Q is negated
  const uint8_t* data;
  CacheGeom g;
  void* o;
  int64_t ld_o;
  int o_bf16;
  float *lse, *part_o, *part_ml;                             // parts: [split][row][head][D], [split][row][head][2]
  int splits, chunk, row_tiles;
};

constexpr float kInf = __builtin_inff();
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

// Eight weights of one row, 2^(scale x - base), as the bf16 terms of an operand; their sum.  A term is the rounded rest that the
// terms before it leave: three hold all 24 bits.
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

// The tokens that a tile of rows and one split go over: [begin, end), begin a multiple of 32
struct Span {
  int begin, end;
  __device__ __forceinline__ Span(const AttnArgs& a, const Sequence& s, int row, int rows, int split) {   // rows > 0
    const int i0 = row / a.group, i1 = (row + rows - 1) / a.group;
    const int hi = s.last(a, i1) + 1, lo = s.first(a, i0) & ~31;
    const int64_t b = lo + (int64_t)split * a.chunk;
    begin = b < hi ? (int)b : hi;
    end = split + 1 < a.splits && b + a.chunk < hi ? (int)b + a.chunk : hi;
    if (end < begin) end = begin;
  }
};

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
};

template <int D, int MODE>
__device__ __forceinline__ Block load_block(const uint8_t* rec, const CacheGeom& g, int row, int blk) {
  Block b;
  const int n = row * (D / 32) + blk;
  b.code = *reinterpret_cast<const u32x4*>(rec + n * 16);
  b.scale = rec[g.scales_at + n];
  b.index = MODE >= 1 ? rec[g.index_at + n] : 0u;
  return b;
}

// 32 bf16 at dst (16-byte aligned, in LDS).  A flushed block, or one to be left out (`drop`), becomes zeros; a scale byte of 255
// makes the unpack-converts answer NaN (also for zero codes, so what is left out gets another).
template <int MODE>
__device__ __forceinline__ void expand(const Block& b, bool drop, uint8_t* dst) {
  const bool zero = drop || b.scale == 0u;
  const uint32_t keep = zero ? 0u : 0xFFFFFFFFu;
  const float X = __uint_as_float((drop ? 127u : b.scale - (MODE == 2 ? b.index >> 5 : 0u)) << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t c = b.code[j] & keep;
    union { bf16x2 v; uint32_t u; } w0, w1, w2, w3;
    w0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 0);
    w1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 1);
    w2.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 2);
    w3.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, X, 3);
    reinterpret_cast<u32x4*>(dst)[j] = u32x4{w0.u, w1.u, w2.u, w3.u};
  }
  if (MODE >= 1) {                                           // 2^e_max * 1.mmm * 2^shared_exp over its element
    const uint32_t pos = b.index & 31u;
    const uint32_t lo = pos & 8u ? b.code[1] : b.code[0], hi = pos & 8u ? b.code[3] : b.code[2];
    const uint32_t nib = ((pos & 16u ? hi : lo) >> (4u * (pos & 7u))) & 15u;
    const uint32_t h = (((nib & 8u) << 12) | ((b.scale + 2u) << 7) | ((nib & 7u) << 4)) & keep;   // (scale byte 255: any number among NaN)
    reinterpret_cast<u16a*>(dst)[pos] = (uint16_t)h;
  }
}

// four tokens (rows `pitch` bytes apart) x 16 channels per 16 lanes, transposed: a lane gets four tokens of one channel
__device__ __forceinline__ s16x4 read_transposed(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t row, int head, int d, f32x4 v) {
  const int64_t off = row * a.ld_o + (int64_t)head * a.g.D + d;
  if (a.o_bf16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + off) = u32x2{bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + off) = v;
}

// The end of a row: the output itself, or this split's part of it
__device__ __forceinline__ void finish_values(const AttnArgs& a, int split, int64_t row, int head, int d, f32x4 v, float l) {
  if (a.splits == 1) store_out(a, row, head, d, l == 0.0f ? f32x4{0, 0, 0, 0} : v / l);
  else *reinterpret_cast<f32x4*>(a.part_o + (((int64_t)split * a.rows + row) * a.heads + head) * a.g.D + d) = v;
}
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f; }
__device__ __forceinline__ void finish_row(const AttnArgs& a, int split, int64_t row, int head, float m, float l) {
  if (a.splits > 1) {
    float* p = a.part_ml + (((int64_t)split * a.rows + row) * a.heads + head) * 2;
    p[0] = m;
    p[1] = l;
  } else if (a.lse) {
    a.lse[row * a.heads + head] = lse_of(m, l);
  }
}

// The work of a workgroup: split fastest, then tile of rows, key-value head, sequence
struct Work {
  int split, tile, head, seq;
  __device__ __forceinline__ explicit Work(const AttnArgs& a) {
    uint32_t id = blockIdx.x;
    split = (int)(id % (uint32_t)a.splits);
    id /= (uint32_t)a.splits;
    tile = (int)(id % (uint32_t)a.row_tiles);
    id /= (uint32_t)a.row_tiles;
    head = (int)(id % (uint32_t)a.g.kv_heads);
    seq = (int)(id / (uint32_t)a.g.kv_heads);
  }
};

// ---- few rows -------------------------------------------------------------------------------------------------------
constexpr int kFewWaves = 4;
template <int D>
constexpr int few_pitch() { return 2 * D + 16; }             // bytes per token: 16 rows' 16-byte reads fall on all banks
template <int D>
constexpr int few_patch(int nt) { return 32 * few_pitch<D>() > 16 * nt * D * 4 ? 32 * few_pitch<D>() : 16 * nt * D * 4; }
template <int D>
constexpr int few_lds(int nt) { return kFewWaves * (few_patch<D>(nt) + 16 * nt * 8); }
constexpr int few_waves_per_simd(int D, int NT) { return D * NT <= 128 ? 4 : D * NT <= 256 ? 2 : 1; }

// NT tiles of 16 rows; TERMS: bf16 terms of P
template <int D, int MODE, int NT, int TERMS>
__global__ void __launch_bounds__(64 * kFewWaves, few_waves_per_simd(D, NT)) attn_few_kernel(const AttnArgs a) {
  constexpr int DB = D / 32, NB = D / 64, PITCH = few_pitch<D>(), PATCH = few_patch<D>(NT);   // blocks per token; per lane of a 32-token tile
  constexpr int LANE_TOKENS = D == 64 ? 32 : 16;             // tokens that a wavefront's lanes cover with one block each (of 2, 4, 4 neighbours)
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  uint8_t* const patch = lds + wave * PATCH;                 // a tile's keys, then its values
  float* const ml = reinterpret_cast<float*>(lds + kFewWaves * PATCH);   // [wave][row][2]
  const Work w(a);
  const Sequence s(a, w.seq);
  const int R = s.n * a.group;
  // this lane's blocks of a tile: its token (16 lanes in a row have 16 tokens: their stores fall on all banks), its block of the token
  const auto token_of = [&](int i) { return D == 256 ? 16 * (i >> 1) + (lane & 15) : LANE_TOKENS * i + (lane & (LANE_TOKENS - 1)); };
  const auto block_of = [&](int i) { return D == 256 ? 4 * (i & 1) + (lane >> 4) : lane / LANE_TOKENS; };
  for (int r0 = w.tile * 16 * NT; r0 < R; r0 += a.row_tiles * 16 * NT) {
    const Span span(a, s, r0, R - r0 < 16 * NT ? R - r0 : 16 * NT, w.split);
    // this lane's rows, as operands of the first product: channels 32 st + 8 quarter ... + 7
    Operand q[NT][DB];
    int first[NT], last[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = r0 + 16 * t + col, i = r / a.group;
      const bool there = r < R;
      first[t] = there ? s.first(a, i) : 1;
      last[t] = there ? s.last(a, i) : 0;
      const uint16_t* p = a.q + (s.q0 + (there ? i : 0)) * a.ld_q + (int64_t)(w.head * a.group + (there ? r - i * a.group : 0)) * D + 8 * quarter;
#pragma unroll
      for (int st = 0; st < DB; ++st) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + 32 * st);
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
    // The wavefront's tiles: span.begin + 32 wave, and every 32 kFewWaves tokens from there.  Lane n holds the page of half n % 2 of
    // tile n / 2 of the next 32 tiles (-1: none), so that a tile's addresses wait for no table.
    const int begin = span.begin + 32 * wave;
    int tile = 0;
    int32_t pages = -1;
    Block kb[NB], vb[NB];
    bool held0 = false, held1 = false;                       // whether the tile's two halves have a page
    const auto fetch = [&](int t) {
      if ((tile & 31) == 0) pages = page_of(a, s, (int64_t)t + 32 * kFewWaves * (lane >> 1) + 16 * (lane & 1));
      const Page p0(a, w.head, __builtin_amdgcn_readlane(pages, 2 * (tile & 31)), t), p1(a, w.head, __builtin_amdgcn_readlane(pages, 2 * (tile & 31) + 1), t + 16);
      held0 = p0.held;
      held1 = p1.held;
      ++tile;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int token = token_of(i);
        const bool second = D == 64 ? token >= 16 : i >= NB / 2;
        const uint8_t* rec = second ? p1.rec : p0.rec;
        const int row = second ? p1.at + (token & 15) : p0.at + token;
        kb[i] = load_block<D, MODE>(rec, a.g, row, block_of(i));
        vb[i] = load_block<D, MODE>(rec + a.g.part_bytes, a.g, row, block_of(i));
      }
    };
    if (begin < span.end) fetch(begin);
    for (int t0 = begin; t0 < span.end; t0 += 32 * kFewWaves) {
      const bool h0 = held0, h1 = held1;
      uint64_t nan[NB];                                      // lanes whose block of V is NaN: zeros here, put in behind the product
      uint64_t any = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) expand<MODE>(kb[i], false, patch + token_of(i) * PITCH + block_of(i) * 64);
      __builtin_amdgcn_wave_barrier();
      f32x4 sc[NT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][h] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < DB; ++st) {
          Operand k;
          const u32x4 x = *reinterpret_cast<const u32x4*>(patch + (16 * h + col) * PITCH + (32 * st + 8 * quarter) * 2);
#pragma unroll
          for (int j = 0; j < 4; ++j) k.u[j] = x[j];
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v, q[t][st].v, sc[t][h], 0, 0, 0);
        }
      }
      __builtin_amdgcn_wave_barrier();                       // (the reads above come first: LDS serves a wavefront in order)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int token = token_of(i);
        const bool dead = t0 + token >= span.end || !(token >= 16 ? h1 : h0);
        nan[i] = __ballot(vb[i].scale == 255u && !dead);
        any |= nan[i];
        expand<MODE>(vb[i], dead || vb[i].scale == 255u, patch + token * PITCH + block_of(i) * 64);
      }
      __builtin_amdgcn_wave_barrier();
      if (t0 + 32 * kFewWaves < span.end) fetch(t0 + 32 * kFewWaves);
      const bool whole = h0 && h1 && t0 >= all_from && t0 + 31 <= all_to && t0 + 32 <= span.end;   // (uniform)
      if (!whole) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = t0 + 16 * h + 4 * quarter + i;
              sc[t][h][i] = tok >= first[t] && tok <= last[t] && tok < span.end && (h ? h1 : h0) ? sc[t][h][i] : -kInf;
            }
      }
      Operand p[NT][TERMS];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float mx = fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), fmaxf(sc[t][0][2], sc[t][0][3])), fmaxf(fmaxf(sc[t][1][0], sc[t][1][1]), fmaxf(sc[t][1][2], sc[t][1][3])));
        mx = fmaxf(m[t], max_across_32(max_across_16(mx)));
        const float base = zero_if_none(mx) * a.scale;
        if (__any(mx != m[t])) {
          const float f = exp2_of(m[t] * a.scale - base);
          l[t] *= f;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) o[t][d] *= f;
          m[t] = mx;
        }
        l[t] += weights<TERMS>(sc[t][0], sc[t][1], a.scale, base, p[t]);
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        Operand v;
        const uint8_t* at = patch + (4 * quarter + (col >> 2)) * PITCH + (16 * d + 4 * (col & 3)) * 2;
        v.s[0] = read_transposed(at);
        v.s[1] = read_transposed(at + 16 * PITCH);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int c = 0; c < TERMS; ++c) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, p[t][c].v, o[t][d], 0, 0, 0);
      }
      if (any) {                                             // NaN blocks of V, for the rows that see them
#pragma unroll
        for (int i = 0; i < NB; ++i)
          for (uint64_t left = nan[i]; left; left &= left - 1) {
            const int who = __builtin_ctzll(left), tok = t0 + __builtin_amdgcn_readlane(token_of(i), who), blk = __builtin_amdgcn_readlane(block_of(i), who);
#pragma unroll
            for (int t = 0; t < NT; ++t)
              if (tok >= first[t] && tok <= last[t]) {
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
                  if (d / 2 == blk) o[t][d] = f32x4{1, 1, 1, 1} * __uint_as_float(0x7FC00000u);
              }
          }
      }
      __builtin_amdgcn_wave_barrier();
    }
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
    for (int j = threadIdx.x; j < 16 * NT * (D / 4); j += 64 * kFewWaves) {
      const int row = j / (D / 4), d = (j - row * (D / 4)) * 4, r = r0 + row;
      if (r >= R) break;
      float top = -kInf, sum = 0.0f;
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) top = fmaxf(top, ml[(v * 16 * NT + row) * 2]);
      const float base = zero_if_none(top);
      f32x4 out = {0, 0, 0, 0};
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) {
        const float f = exp2_of(ml[(v * 16 * NT + row) * 2] - base);
        sum += ml[(v * 16 * NT + row) * 2 + 1] * f;
        out += *reinterpret_cast<const f32x4*>(lds + v * PATCH + (row * D + d) * 4) * f;
      }
      const int i = r / a.group, head = w.head * a.group + r - i * a.group;
      finish_values(a, w.split, s.q0 + i, head, d, out, sum);
      if (d == 0) finish_row(a, w.split, s.q0 + i, head, top, sum);
    }
    __syncthreads();
  }
}

// ---- many rows ------------------------------------------------------------------------------------------------------
constexpr int kManyWaves = 4, kManyTokens = 64, kManyRows = 32 * kManyWaves;
template <int D>
constexpr int many_pitch() { return 2 * D + 16; }
template <int D>
constexpr int many_buffers() { return D == 256 ? 1 : 2; }    // (two of D = 256 exceed the 160 KiB of a compute unit together with nothing else)
template <int D>
constexpr int many_lds() { return many_buffers<D>() * 2 * kManyTokens * many_pitch<D>() + 2 * kManyWaves * 2 * 4 * 8; }

template <int D, int MODE, int TERMS>
__global__ void __launch_bounds__(64 * kManyWaves) attn_many_kernel(const AttnArgs a) {
  constexpr int DB = D / 32, NB = kManyTokens * DB / (64 * kManyWaves), PITCH = many_pitch<D>();
  constexpr int BUF = many_buffers<D>(), HALF = kManyTokens * PITCH;
  static_assert(NB * 64 * kManyWaves == kManyTokens * DB || D == 64, "blocks per lane");
  constexpr int NL = NB < 1 ? 1 : NB;                        // D = 64: 128 blocks, the upper wavefronts have none
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  uint64_t* const nans = reinterpret_cast<uint64_t*>(lds + BUF * 2 * HALF);   // [buffer][wave][NL] lanes with a NaN block of V
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const Work w(a);
  const Sequence s(a, w.seq);
  const int R = s.n * a.group, tiles = (R + kManyRows - 1) / kManyRows;
  for (int turn = w.tile; turn < tiles; turn += a.row_tiles) {
    const int r0 = (tiles - 1 - turn) * kManyRows;           // the last rows see most: they start first
    const Span span(a, s, r0, R - r0 < kManyRows ? R - r0 : kManyRows, w.split);
    const int r = r0 + 32 * wave + col, i = r / a.group;
    const bool there = r < R;
    const int first = there ? s.first(a, i) : 1, last = there ? s.last(a, i) : 0;
    const int head = w.head * a.group + (there ? r - i * a.group : 0);
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
    Block kb[NL], vb[NL];
    uint32_t held = 0, held_next = 0;                        // bit j: tokens 16 j ... + 15 of the tile have a page
    int tile = 0;
    int32_t pages = -1;                                      // lane n: the page of tokens 16 (n % 4) ... of tile n / 4 of the next 16
    const auto fetch = [&](int t) {
      if ((tile & 15) == 0) pages = page_of(a, s, (int64_t)t + 16 * lane);
      held_next = 0;
      const uint8_t* rec[4];
      int at[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Page p(a, w.head, __builtin_amdgcn_readlane(pages, 4 * (tile & 15) + j), t + 16 * j);
        held_next |= (p.held ? 1u : 0u) << j;
        rec[j] = p.rec;
        at[j] = p.at;
      }
      ++tile;
#pragma unroll
      for (int k = 0; k < NL; ++k) {
        const int n = (int)threadIdx.x + 64 * kManyWaves * k, token = n / DB;
        if (token < kManyTokens) {
          const int j = token >> 4;
          const uint8_t* base = j & 2 ? (j & 1 ? rec[3] : rec[2]) : (j & 1 ? rec[1] : rec[0]);
          const int row = (j & 2 ? (j & 1 ? at[3] : at[2]) : (j & 1 ? at[1] : at[0])) + (token & 15);
          kb[k] = load_block<D, MODE>(base, a.g, row, n % DB);
          vb[k] = load_block<D, MODE>(base + a.g.part_bytes, a.g, row, n % DB);
        }
      }
    };
    const auto expand_all = [&](int t, int buf) {            // the fetched tile into a buffer
      uint8_t* const kt = lds + buf * 2 * HALF;
#pragma unroll
      for (int k = 0; k < NL; ++k) {
        const int n = (int)threadIdx.x + 64 * kManyWaves * k, token = n / DB;
        bool bad = false;
        if (token < kManyTokens) {
          const bool dead = t + token >= span.end || !((held_next >> (token >> 4)) & 1u);
          expand<MODE>(kb[k], false, kt + token * PITCH + (n % DB) * 64);
          bad = vb[k].scale == 255u && !dead;
          expand<MODE>(vb[k], dead || bad, kt + HALF + token * PITCH + (n % DB) * 64);
        }
        const uint64_t b = __ballot(bad);
        if (lane == 0) nans[(buf * kManyWaves + wave) * NL + k] = b;
      }
    };
    int buf = 0;
    if (span.begin < span.end) {
      fetch(span.begin);
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
            const u32x4 x = *reinterpret_cast<const u32x4*>(kt + (32 * h + col) * PITCH + (16 * st + 8 * half) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) k.u[j] = x[j];
            sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.v, q[st].v, sc[h], 0, 0, 0);
          }
        }
        const bool whole = held == 15u && t0 >= all_from && t0 + kManyTokens - 1 <= all_to && t0 + kManyTokens <= span.end;
        if (!whole) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int tok = t0 + 32 * h + 8 * (j >> 2) + 4 * half + (j & 3);
              sc[h][j] = tok >= first && tok <= last && tok < span.end && ((held >> (2 * h + (j >> 3))) & 1u) ? sc[h][j] : -kInf;
            }
        }
        float mx = -kInf;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 16; ++j) mx = fmaxf(mx, sc[h][j]);
        mx = fmaxf(m, max_across_32(mx));
        const float base = zero_if_none(mx) * a.scale;
        if (__any(mx != m)) {
          const float f = exp2_of(m * a.scale - base);
          l *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d] *= f;
          m = mx;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {                        // 16 tokens: registers 8 (b % 2) ... + 7 of half b / 2
          Operand p[TERMS];
          const int j = 8 * (b & 1);
          const f32x16& x = sc[b >> 1];
          l += weights<TERMS>(f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]}, f32x4{x[j + 4], x[j + 5], x[j + 6], x[j + 7]}, a.scale, base, p);
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            Operand v;
            const uint8_t* at = vt + (16 * b + 4 * half + ((lane & 15) >> 2)) * PITCH + (32 * d + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
            v.s[0] = read_transposed(at);
            v.s[1] = read_transposed(at + 8 * PITCH);
#pragma unroll
            for (int c = 0; c < TERMS; ++c) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, p[c].v, o[d], 0, 0, 0);
          }
        }
        uint64_t any = 0;
#pragma unroll
        for (int k = 0; k < kManyWaves * NL; ++k) any |= nans[buf * kManyWaves * NL + k];
        if (__any(any != 0)) {                               // NaN blocks of V, for the rows that see them
          for (int k = 0; k < kManyWaves * NL; ++k)
            for (uint64_t left = nans[buf * kManyWaves * NL + k]; left; left &= left - 1) {
              const int n = __builtin_ctzll(left) + 64 * (k / NL) + 64 * kManyWaves * (k % NL), tok = t0 + n / DB;
              if (tok >= first && tok <= last) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
                  if (d == n % DB)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[d][j] = __uint_as_float(0x7FC00000u);
              }
            }
        }
      }
      if (more) {
        if (BUF == 1) __syncthreads();                       // everyone is done with the only buffer
        else buf ^= 1;
        expand_all(t0 + kManyTokens, buf);
      }
    }
    l = sum_across_32(l);
    if (there) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          finish_values(a, w.split, s.q0 + i, head, 32 * d + 8 * j + 4 * half, f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]}, l);
      if (half == 0) finish_row(a, w.split, s.q0 + i, head, m * a.scale, l);
    }
    __syncthreads();
  }
}

// ---- the parts of split sequences ---------------------------------------------------------------------------------------
// A workgroup per (row, head): every lane the weight of one part (at most kMostSplits = lanes), then D / 4 lanes across a row and
// 1024 / D parts at a time.  Rows that no sequence has are left as they are.
constexpr int kMostSplits = 256;
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnArgs a) {
  __shared__ float weight[kMostSplits], top_of[4], sum_of[4];
  __shared__ __attribute__((aligned(16))) float acc[1024];
  const int t = threadIdx.x, across = a.g.D >> 2, d = 4 * (t & (across - 1)), g = t / across, groups = 256 / across;
  const int64_t from = a.q_start ? a.q_start[0] : 0, to = a.q_start ? a.q_start[a.n_seq] : a.rows, n = a.rows * a.heads;
  for (int64_t j = blockIdx.x; j < n; j += gridDim.x) {
    const int64_t row = j / a.heads;
    if (row < from || row >= to) continue;                   // (the whole workgroup)
    const int head = (int)(j - row * a.heads);
    float m = -kInf, l = 0.0f;
    if (t < a.splits) {
      m = a.part_ml[(t * n + j) * 2];
      l = a.part_ml[(t * n + j) * 2 + 1];
    }
    float top = m;
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    if ((t & 63) == 0) top_of[t >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
    const float f = l == 0.0f ? 0.0f : exp2_of(m - zero_if_none(top));   // (0: a part that saw nothing, left out below)
    weight[t] = f;
    float sum = l * f;
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
    if ((t & 63) == 0) sum_of[t >> 6] = sum;
    __syncthreads();
    sum = (sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]);
    f32x4 out = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = g; p < a.splits; p += groups) {
      const float w = weight[p];
      const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + (p * n + j) * a.g.D + d);
      if (w != 0.0f) out += x * w;
    }
    *reinterpret_cast<f32x4*>(acc + 4 * t) = out;
    __syncthreads();
    if (g == 0) {
      for (int p = 1; p < groups; ++p) out += *reinterpret_cast<const f32x4*>(acc + 4 * (t + p * across));
      store_out(a, row, head, d, sum == 0.0f ? f32x4{0, 0, 0, 0} : out / sum);
    }
    if (t == 0 && a.lse) a.lse[row * a.heads + head] = lse_of(top, sum);
    __syncthreads();
  }
}

// ---- launch -----------------------------------------------------------------------------------------------------------
struct Plan {
  bool many;
  int nt, row_tiles, splits, chunk;
  int64_t wgs;
};

// Which kernel, and over how many workgroups a sequence's tokens are split.  Up to 32 rows of a key-value head: attn_few_kernel.
Plan plan_for(int64_t n_seq, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads, int64_t window) {
  Plan p;
  const int64_t rows = max_q * (heads / kv_heads);           // of one key-value head
  p.many = rows > 32;
  p.nt = rows > 16 ? 2 : 1;
  const int64_t tile = p.many ? kManyRows : 16 * p.nt;
  p.row_tiles = (int)((rows + tile - 1) / tile);
  if (p.row_tiles < 1) p.row_tiles = 1;
  const int64_t base = n_seq * kv_heads * p.row_tiles;
  // tokens that one tile of rows goes over, at most
  int64_t len = max_kv;
  if (window > 0 && window + max_q + 32 < len) len = window + max_q + 32;
  const int64_t least = p.many ? 512 : 256, want = 1024;     // tokens per workgroup at least; workgroups wanted
  int64_t splits = base < want ? (want + base - 1) / base : 1;
  if (splits > (len + least - 1) / least) splits = (len + least - 1) / least;
  if (splits < 1) splits = 1;
  if (splits > kMostSplits) splits = kMostSplits;
  const int64_t step = p.many ? kManyTokens : 32 * kFewWaves;
  const int64_t chunk = ((len + splits - 1) / splits + step - 1) / step * step;
  p.chunk = (int)(chunk < step ? step : chunk > (1 << 30) ? (1 << 30) : chunk);
  p.splits = (int)((len + p.chunk - 1) / p.chunk);
  if (p.splits < 1) p.splits = 1;
  p.wgs = base * p.splits;
  return p;
}

size_t parts_bytes(const Plan& p, int64_t rows, int64_t heads, int64_t D) {
  return p.splits > 1 ? (size_t)p.splits * (size_t)rows * (size_t)heads * (size_t)(D + 2) * 4 : 0;
}

template <int D, int MODE, int TERMS>
void launch(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const dim3 grid((unsigned)p.wgs);
  if (p.many) {
    allow_dynamic_lds<attn_many_kernel<D, MODE, TERMS>>(many_lds<D>());
    hipLaunchKernelGGL((attn_many_kernel<D, MODE, TERMS>), grid, dim3(64 * kManyWaves), many_lds<D>(), s, a);
  } else if (p.nt == 2) {
    allow_dynamic_lds<attn_few_kernel<D, MODE, 2, TERMS>>(few_lds<D>(2));
    hipLaunchKernelGGL((attn_few_kernel<D, MODE, 2, TERMS>), grid, dim3(64 * kFewWaves), few_lds<D>(2), s, a);
  } else {
    allow_dynamic_lds<attn_few_kernel<D, MODE, 1, TERMS>>(few_lds<D>(1));
    hipLaunchKernelGGL((attn_few_kernel<D, MODE, 1, TERMS>), grid, dim3(64 * kFewWaves), few_lds<D>(1), s, a);
  }
}

// shape rules that the size function and the call share
bool shapes_fit(int64_t n_seq, int64_t rows, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads) {
  return n_seq >= 0 && rows >= 0 && max_q >= 0 && max_kv >= 0 && heads >= 1 && heads <= 65535 && kv_heads >= 1 && heads % kv_heads == 0 &&
         rows <= 2147483647LL && max_q <= 2147483647LL && max_kv <= 2147483647LL && n_seq <= 2147483647LL;
}

}  // namespace

extern "C" size_t mxp_attention_workspace_bytes(int64_t n_seq, int64_t rows, int64_t max_q, int64_t max_kv, int64_t heads, int64_t kv_heads,
                                                int64_t head_dim, int64_t window) {
  if (!shapes_fit(n_seq, rows, max_q, max_kv, heads, kv_heads) || n_seq == 0 || rows == 0 || rows * heads > kMostRows || head_dim < 1 || window < 0) return 0;
  return parts_bytes(plan_for(n_seq, max_q < rows ? max_q : rows, max_kv, heads, kv_heads, window), rows, heads, head_dim);
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
  const Plan p = plan_for(n_seq, max_q < rows ? max_q : rows, max_kv, heads, kv_heads, window);
  if (p.wgs > 2147483647LL) return MXP_ERR_UNSUPPORTED;
  const size_t need = parts_bytes(p, rows, heads, head_dim);
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
  if (a.scale < 1.17549435e-38f) a.scale = 1.17549435e-38f;   // (0 would make NaN of a hidden token's -infinity)
  a.flip = scale < 0 ? 0x80008000u : 0u;
  a.data = static_cast<const uint8_t*>(cache);
  a.o = O;
  a.ld_o = ld_o;
  a.o_bf16 = o_dtype == MXP_BF16;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = need ? a.part_o + (size_t)p.splits * rows * heads * head_dim : nullptr;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.row_tiles = p.row_tiles;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define MXP_ATTN_T(D, M) do { if (a.o_bf16) launch<D, M, 1>(a, p, s); else launch<D, M, 3>(a, p, s); } while (0)
#define MXP_ATTN_M(D) do { if (fmt == MXP_FMT_MXFP4) MXP_ATTN_T(D, 0); else if (fmt == MXP_FMT_MXFP4P) MXP_ATTN_T(D, 1); else MXP_ATTN_T(D, 2); } while (0)
  if (head_dim == 64) MXP_ATTN_M(64);
  else if (head_dim == 128) MXP_ATTN_M(128);
  else MXP_ATTN_M(256);
#undef MXP_ATTN_M
#undef MXP_ATTN_T
  if (p.splits > 1) {
    const int64_t want = rows * heads;
    hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)(want < (1 << 20) ? want : (1 << 20))), dim3(256), 0, s, a);
  }
  return launch_status();
}
