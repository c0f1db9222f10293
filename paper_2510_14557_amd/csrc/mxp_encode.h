// Device code of the conversion of one block (Sec. 4.1, 4.2, Eq. 1), shared by the kernels that write block formats.  Four
// lanes (a quad) share a block of 32, a lane holds 8 consecutive elements.
#pragma once
#include "mxp_common.h"

namespace mxp {

typedef __bf16 enc_v2bf __attribute__((ext_vector_type(2)));
typedef short enc_v2s __attribute__((ext_vector_type(2)));
typedef __bf16 enc_v32bf __attribute__((ext_vector_type(32)));
typedef float enc_v16f __attribute__((ext_vector_type(16)));
typedef uint32_t enc_v6u __attribute__((ext_vector_type(6)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_mov(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kQuadSwap1 = 0xB1;  // quad_perm [1,0,3,2]
constexpr int kQuadSwap2 = 0x4E;  // quad_perm [2,3,0,1]
constexpr int kQuadFromEven = 0xA0;  // quad_perm [0,0,2,2]: odd lanes read their left neighbour
constexpr int kRowShr4 = 0x114;
constexpr int kRowShr8 = 0x118;

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// 3-bit BM mantissa from the 23-bit fraction of the block maximum: round to nearest even on bit 20, and a carry
// out of the field saturates (the shared scale is never altered, Sec. 4.1).
__device__ __forceinline__ uint32_t bm_mantissa(uint32_t frac23) {
  uint32_t m = (frac23 + 0x7FFFFu + ((frac23 >> 20) & 1u)) >> 20;
  return umin(m, 7u);
}

// One group = 8 consecutive elements of one block, held by one lane.  `part` = which quarter of the block.
// Returns the packed dword of 8 nibbles; scale byte and index byte are returned in all four lanes of the quad.
// MODE: 0 = MXFP4, 1 = MXFP4+, 2 = MXFP4++ (Sec. 4.3: the NBMs are scaled by 2^(shared_exp - delta), where
// shared_exp - delta = CLIP(largest NBM exponent - e_max + 1, {shared_exp - 7, shared_exp}), and delta goes into bits
// 7:5 of the index byte; delta is also kept <= scale byte - 1 so that the NBM scale stays an E8M0 number).
template <bool BF16, int MODE>
__device__ __forceinline__ uint32_t encode_group(const uint32_t (&w)[8], int part, uint32_t& sbyte, uint32_t& idx) {
  constexpr bool PLUS = MODE >= 1, PP = MODE == 2;
  uint32_t amax32;  // magnitude bits of the block maximum, as an fp32 pattern
  uint32_t a2 = 0;  // (PP) magnitude bits of the largest element other than the BM
  if (BF16) {
    // key = magnitude(15 bit) << 16 | (31 - position): one unsigned max gives the maximum and, among equal
    // magnitudes, the lowest position.
    uint32_t k = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t m = w[j] & 0x7FFF7FFFu;
      uint32_t klo = (m << 16) | (uint32_t)(7 - 2 * j);
      uint32_t khi = (m & 0xFFFF0000u) | (uint32_t)(6 - 2 * j);
      k = umax(k, umax(klo, khi));
    }
    k += (uint32_t)(3 - part) * 8u;
    k = umax(k, dpp_mov<kQuadSwap1>(k));
    k = umax(k, dpp_mov<kQuadSwap2>(k));
    amax32 = k & 0xFFFF0000u;
    idx = 31u - (k & 31u);
    if (PP) {
      // keys are unique (the position is part of them): the lane whose best key won leaves that element out
      uint32_t k2 = 0;
      const uint32_t off = (uint32_t)(3 - part) * 8u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t m = w[j] & 0x7FFF7FFFu;
        const uint32_t klo = ((m << 16) | (uint32_t)(7 - 2 * j)) + off;
        const uint32_t khi = ((m & 0xFFFF0000u) | (uint32_t)(6 - 2 * j)) + off;
        k2 = umax(k2, klo == k ? 0u : klo);
        k2 = umax(k2, khi == k ? 0u : khi);
      }
      k2 = umax(k2, dpp_mov<kQuadSwap1>(k2));
      k2 = umax(k2, dpp_mov<kQuadSwap2>(k2));
      a2 = k2 & 0xFFFF0000u;
    }
  } else {
    uint32_t a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = w[i] & 0x7FFFFFFFu;
    uint32_t mx = a[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = umax(mx, a[i]);
    mx = umax(mx, dpp_mov<kQuadSwap1>(mx));
    mx = umax(mx, dpp_mov<kQuadSwap2>(mx));
    uint32_t p = 32u;
#pragma unroll
    for (int i = 7; i >= 0; --i) p = (a[i] == mx) ? (uint32_t)(part * 8 + i) : p;
    p = umin(p, dpp_mov<kQuadSwap1>(p));
    p = umin(p, dpp_mov<kQuadSwap2>(p));
    amax32 = mx;
    idx = p;
    if (PP) {
      uint32_t m2 = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m2 = umax(m2, (uint32_t)(part * 8 + i) == p ? 0u : a[i]);
      m2 = umax(m2, dpp_mov<kQuadSwap1>(m2));
      m2 = umax(m2, dpp_mov<kQuadSwap2>(m2));
      a2 = m2;
    }
  }
  const uint32_t E = amax32 >> 23;                     // biased exponent of the BM = floor(log2) + 127
  const bool flush = E <= 2u;                          // floor(log2 BM) <= -127 + e_max      (Sec. 4.1)
  const bool nonfinite = E == 255u;
  uint32_t delta = 0;
  if (PP) {
    const uint32_t sb = E - 2u, E2 = a2 >> 23;                       // biased: BM scale; exponent of the largest NBM
    const uint32_t lo = sb > 7u ? sb - 7u : 0u;                      // (flushed blocks are reset below)
    uint32_t nb = E2 == 0u ? lo : umin(umax(E2 - 1u, lo), sb);       // biased shared_exp_new = E2 - 127 - e_max + 1 + 127
    nb = umax(nb, 1u);
    delta = sb - nb;
  }
  // X = 2^shared_exp, shared_exp = floor(log2 BM) - e_max (Eq. 1); the NBMs of MXFP4++ use 2^(shared_exp - delta)
  const float scale = __uint_as_float((E - 2u - delta) << 23);
  uint32_t packed = 0;
  if (BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      union { uint32_t u; enc_v2bf v; } c;
      c.u = w[j];
      if (j == 0) packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, c.v, scale, 0);
      if (j == 1) packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, c.v, scale, 1);
      if (j == 2) packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, c.v, scale, 2);
      if (j == 3) packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, c.v, scale, 3);
    }
  } else {
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, __uint_as_float(w[4]), __uint_as_float(w[5]), scale, 2);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, __uint_as_float(w[6]), __uint_as_float(w[7]), scale, 3);
  }
  if (PLUS) {
    // BM nibble = sign | m2 m1 m0 ; the sign is already in the converted nibble.
    const uint32_t m3 = bm_mantissa(amax32 & 0x7FFFFFu);
    const uint32_t sh = (idx & 7u) * 4u;
    const uint32_t nib = ((packed >> sh) & 8u) | m3;
    const uint32_t repl = (packed & ~(0xFu << sh)) | (nib << sh);
    packed = ((idx >> 3) == (uint32_t)part) ? repl : packed;
  }
  sbyte = E - 2u;
  if (PP) idx |= delta << 5;
  if (flush || nonfinite) {
    packed = 0;
    idx = 0;
    sbyte = nonfinite ? 255u : 0u;
  }
  return packed;
}

// ---- six- and eight-bit elements ------------------------------------------------------------------------------------
template <int BITS>
struct Elem;
template <>
struct Elem<6> {   // E2M3
  static constexpr int MB = 3, BIAS = 1, EMAX = 2;
  static constexpr uint32_t MAXCODE = 0x1Fu;   // 7.5
};
template <>
struct Elem<8> {   // E4M3 (OCP): S.1111.111 is NaN, the largest number is S.1111.110 = 448
  static constexpr int MB = 3, BIAS = 7, EMAX = 8;
  static constexpr uint32_t MAXCODE = 0x7Eu;
};

// Round-to-nearest-even of sig >> shift, 1 <= shift <= 31.
__device__ __forceinline__ uint32_t rne_shift(uint32_t sig, uint32_t shift) {
  const uint32_t t = sig >> shift, rem = sig & ((1u << shift) - 1u), half = 1u << (shift - 1u);
  return t + ((rem > half || (rem == half && (t & 1u))) ? 1u : 0u);
}

// Magnitude code of an ordinary element: a = fp32 magnitude bits of x, the block scale is 2^(sbyte - 127).
// exponent/mantissa fields are produced as one integer, so a mantissa carry moves into the exponent by itself and
// the subnormal range (field 0) needs no case of its own beyond its larger shift.
template <int BITS>
__device__ __forceinline__ uint32_t elem_code(uint32_t a, int sbyte) {
  using F = Elem<BITS>;
  if (a == 0u) return 0u;
  int ea = (int)(a >> 23);
  uint32_t sig = a & 0x7FFFFFu;
  if (ea == 0) {                       // fp32 subnormal input: normalise so that bit 23 is the leading one
    const int lz = __builtin_clz(sig) - 8;
    sig <<= lz;
    ea = 1 - lz;
  } else {
    sig |= 0x800000u;
  }
  const int t = ea - sbyte + F::BIAS;  // exponent field the scaled value would have as a normal number
  const int eff = t > 1 ? t : 1;
  int shift = (23 - F::MB) + (eff - t);
  shift = shift > 31 ? 31 : shift;     // sig < 2^24: everything beyond 25 rounds to zero anyway
  const uint32_t code = ((uint32_t)(eff - 1) << F::MB) + rne_shift(sig, (uint32_t)shift);
  return umin(code, F::MAXCODE);
}

// BM mantissa of a + format: FB = BITS - 1 fraction bits at exponent e_max; a carry out of the field saturates (the
// shared scale is never altered, Sec. 4.1).  The BM of a block that is not flushed is a normal fp32 number.
template <int BITS>
__device__ __forceinline__ uint32_t bm_code(uint32_t a) {
  constexpr int FB = BITS - 1;
  return umin(rne_shift(a & 0x7FFFFFu, 23 - FB), (1u << FB) - 1u);
}

// One lane's 8 elements of a six- or eight-bit block.  raw: as loaded (4 dwords of bf16 pairs or 8 of fp32); a, sg: magnitude
// bits as an fp32 pattern, sign.  lo, hi: its 48 or 64 code bits; scale and index byte are returned in all four lanes.
template <bool BF16, int BITS, bool PLUS>
__device__ __forceinline__ void encode_wide_group(const uint32_t (&raw)[8], const uint32_t (&a)[8], const uint32_t (&sg)[8], uint32_t part,
                                                  uint32_t& lo, uint32_t& hi, uint32_t& sb, uint32_t& idx) {
  using F = Elem<BITS>;
  uint32_t mx = a[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = umax(mx, a[i]);
  mx = umax(mx, dpp_mov<kQuadSwap1>(mx));
  mx = umax(mx, dpp_mov<kQuadSwap2>(mx));
  uint32_t pos = 32u;                             // lowest position holding the maximum
#pragma unroll
  for (int i = 7; i >= 0; --i) pos = (a[i] == mx) ? part * 8u + (uint32_t)i : pos;
  pos = umin(pos, dpp_mov<kQuadSwap1>(pos));
  pos = umin(pos, dpp_mov<kQuadSwap2>(pos));
  const uint32_t E = mx >> 23;
  const bool flush = E <= (uint32_t)F::EMAX, nonfinite = E == 255u;
  const int sbyte = (int)E - F::EMAX;             // Eq. 1
  lo = hi = 0;                                    // this lane's code bits: 48 (lo, hi[15:0]) or 64
  if (BITS == 8) {
    // E4M3 elements: the CDNA4 pack-convert (x / X, round to nearest even, sign kept), two per instruction; the BM
    // byte of a + format is replaced afterwards
    const float X = __uint_as_float((uint32_t)(sbyte > 0 ? sbyte : 1) << 23);
    enc_v2s plo = {0, 0}, phi = {0, 0};
    if (BF16) {
      union { uint32_t u; enc_v2bf v; } c0, c1, c2, c3;
      c0.u = raw[0]; c1.u = raw[1]; c2.u = raw[2]; c3.u = raw[3];
      plo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(plo, c0.v, X, false);
      plo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(plo, c1.v, X, true);
      phi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(phi, c2.v, X, false);
      phi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(phi, c3.v, X, true);
    } else {
      plo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(plo, __uint_as_float(raw[0]), __uint_as_float(raw[1]), X, false);
      plo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(plo, __uint_as_float(raw[2]), __uint_as_float(raw[3]), X, true);
      phi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(phi, __uint_as_float(raw[4]), __uint_as_float(raw[5]), X, false);
      phi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(phi, __uint_as_float(raw[6]), __uint_as_float(raw[7]), X, true);
    }
    union { enc_v2s v; uint32_t u; } ul, uh;
    ul.v = plo;
    uh.v = phi;
    // the instruction answers magnitudes that round above 448 with the NaN code S.1111.111; the format saturates:
    // clear bit 0 of every byte whose low seven bits are all ones
    lo = ul.u & ~((((ul.u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7);
    hi = uh.u & ~((((uh.u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7);
    if (PLUS && (pos >> 3) == part) {
      const uint32_t i = pos & 7u, sh = (i & 3u) * 8u;
      uint32_t ai = 0, si = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ai = i == (uint32_t)k ? a[k] : ai;
        si = i == (uint32_t)k ? sg[k] : si;
      }
      const uint32_t code = bm_code<8>(ai) | (si << 7);
      if (i < 4u) lo = (lo & ~(0xFFu << sh)) | (code << sh);
      else hi = (hi & ~(0xFFu << sh)) | (code << sh);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t c = (PLUS && pos == part * 8u + (uint32_t)i) ? bm_code<BITS>(a[i]) : elem_code<BITS>(a[i], sbyte);
      c |= sg[i] << (BITS - 1);
      const int b = i * BITS;                     // bit position inside the lane's string
      if (b < 32) lo |= c << b;
      if (b + BITS > 32) hi |= (b >= 32) ? (c << (b - 32)) : (c >> (32 - b));
    }
  }
  sb = (uint32_t)sbyte;
  idx = pos;
  if (flush || nonfinite) {
    lo = hi = 0;
    idx = 0;
    sb = nonfinite ? 255u : 0u;
  }
}

// The same for MXFP6 / MXFP6+ through the 32-element pack-convert: every lane of the quad collects the whole block and converts it,
// lanes 0..2 keep 8 of the 24 bytes each (s0, s1; lane 3's are no part of it).  w: as loaded, 4 dwords of bf16 pairs or 8 of fp32.
constexpr int kQuadLane0 = 0x00, kQuadLane1 = 0x55, kQuadLane2 = 0xAA, kQuadLane3 = 0xFF;   // quad_perm broadcasts
template <bool BF16, bool PLUS>
__device__ __forceinline__ void encode_fp6_group(const uint32_t (&w)[BF16 ? 4 : 8], const uint32_t (&a)[8], uint32_t part, uint32_t& s0,
                                                 uint32_t& s1, uint32_t& sb, uint32_t& idx) {
  using F = Elem<6>;
  constexpr int NW = BF16 ? 4 : 8;
  uint32_t mx = a[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = umax(mx, a[i]);
  mx = umax(mx, dpp_mov<kQuadSwap1>(mx));
  mx = umax(mx, dpp_mov<kQuadSwap2>(mx));
  uint32_t pos = 32u;                             // lowest position holding the maximum
#pragma unroll
  for (int i = 7; i >= 0; --i) pos = a[i] == mx ? part * 8u + (uint32_t)i : pos;
  pos = umin(pos, dpp_mov<kQuadSwap1>(pos));
  pos = umin(pos, dpp_mov<kQuadSwap2>(pos));
  const uint32_t E = mx >> 23;
  const bool flush = E <= (uint32_t)F::EMAX, nonfinite = E == 255u;
  const int sbyte = (int)E - F::EMAX;
  const float X = __uint_as_float((uint32_t)(sbyte > 0 ? sbyte : 1) << 23);
  // the whole block in every lane of the quad
  uint32_t all[4 * NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    all[0 * NW + j] = dpp_mov<kQuadLane0>(w[j]);
    all[1 * NW + j] = dpp_mov<kQuadLane1>(w[j]);
    all[2 * NW + j] = dpp_mov<kQuadLane2>(w[j]);
    all[3 * NW + j] = dpp_mov<kQuadLane3>(w[j]);
  }
  enc_v6u r;
  if (BF16) {
    union { uint32_t u[16]; enc_v32bf v; } c;
#pragma unroll
    for (int i = 0; i < 16; ++i) c.u[i] = all[i];
    r = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(c.v, X);
  } else {
    enc_v16f lo16, hi16;
#pragma unroll
    for (int i = 0; i < 16; ++i) {                   // the two sources are interleaved: code 2i from the first, 2i + 1 from the second
      lo16[i] = __uint_as_float(all[2 * i]);
      hi16[i] = __uint_as_float(all[2 * i + 1]);
    }
    r = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(lo16, hi16, X);
  }
  // this lane's share: dwords 2 part, 2 part + 1 (lane 3 stores nothing)
  s0 = part == 0u ? r[0] : (part == 1u ? r[2] : r[4]);
  s1 = part == 0u ? r[1] : (part == 1u ? r[3] : r[5]);
  if (PLUS) {
    // the BM's magnitude mmmmm at bit 6 pos of the block's string = bit rel of this share (may hang over either edge); its
    // sign is there already: a BM is at least 4 X, and the conversion keeps the sign
    const uint32_t code = bm_code<6>(mx);
    const int rel = (int)(6u * pos) - 64 * (int)part;
    uint64_t share = ((uint64_t)s1 << 32) | s0;
    if (rel > -6 && rel < 64) {
      const uint64_t m = rel >= 0 ? ((uint64_t)0x1Fu << rel) : ((uint64_t)0x1Fu >> (-rel));
      const uint64_t c = rel >= 0 ? ((uint64_t)code << rel) : ((uint64_t)code >> (-rel));
      share = (share & ~m) | c;
    }
    s0 = (uint32_t)share;
    s1 = (uint32_t)(share >> 32);
  }
  sb = (uint32_t)sbyte;
  idx = pos;
  if (flush || nonfinite) {
    s0 = s1 = 0;
    idx = 0;
    sb = nonfinite ? 255u : 0u;
  }
}

}  // namespace mxp
