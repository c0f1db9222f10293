// mxp_rmsnorm_quantize: h = x + residual, root-mean-square norm of h, converted to a block format in the same pass.
//
//   h = round(x + r),   y = h * (sum(h^2) / K + eps)^-1/2 * w,   blocks of y -> codes, scales, index (Sec. 4.1, Eq. 1)
//
// HBM-bound: x and r are read once, h and the codes written once, about six flops a value.  A workgroup holds a row in its
// registers between the sum and the conversion (16 values a lane, up to 1024 lanes); a longer row is read a second time.
// 4096 rows of 4096, bf16 -> MXFP8 with residual, 118 MB: 23.8 us (5.0 TB/s, a copy's rate); 1 row 3.5 us, of which a launch alone is 2.3.
#include "mxp_common.h"
#include "mxp_encode.h"

namespace {

using namespace mxp;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct NormArgs {
  const void *x, *r, *w;
  void* h;
  int64_t rows, ld_x, ld_r, ld_h;
  int K, w_bf16;
  float eps;
  uint8_t *elems, *scales, *bm_idx;
};

// eight consecutive values as fp32
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t off, float (&v)[8]) {
  if (BF16) {
    const u32x4 t = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + off);
    const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  } else {
    const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + off);
    const u32x4 a = q[0], b = q[1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  }
}

// x + r in the type of x: the sum is rounded once, and the norm is of what is stored
template <bool BF16>
__device__ __forceinline__ void load_sum(const NormArgs& a, int64_t row, int g, float (&v)[8]) {
  load8<BF16>(a.x, row * a.ld_x + g * 8, v);
  if (a.r) {
    float r[8];
    load8<BF16>(a.r, row * a.ld_r + g * 8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = BF16 ? (float)(__bf16)(v[i] + r[i]) : v[i] + r[i];
  }
}

template <bool BF16>
__device__ __forceinline__ void store8(void* p, int64_t off, const float (&v)[8]) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(v[i]);
  if (BF16) {                                                        // (the values are bf16 numbers)
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + off) =
        u32x4{(b[0] >> 16) | (b[1] & 0xFFFF0000u), (b[2] >> 16) | (b[3] & 0xFFFF0000u), (b[4] >> 16) | (b[5] & 0xFFFF0000u), (b[6] >> 16) | (b[7] & 0xFFFF0000u)};
  } else {
    u32x4* q = reinterpret_cast<u32x4*>(static_cast<float*>(p) + off);
    q[0] = u32x4{b[0], b[1], b[2], b[3]};
    q[1] = u32x4{b[4], b[5], b[6], b[7]};
  }
}

// y of one lane (8 values, a quad of lanes a block) -> its place in the canonical arrays
template <int FMT>
__device__ __forceinline__ void convert_store(const NormArgs& a, int64_t row, int g, const float (&y)[8]) {
  const uint32_t part = threadIdx.x & 3u;
  const int64_t blk = row * (a.K / kBlock) + (g >> 2);
  uint32_t raw[8], sb, idx;
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i] = __float_as_uint(y[i]);
  if constexpr (FMT <= MXP_FMT_MXFP4PP) {
    const uint32_t packed = encode_group<false, FMT>(raw, (int)part, sb, idx);
    reinterpret_cast<uint32_t*>(a.elems)[blk * 4 + part] = packed;
  } else {
    constexpr bool PLUS = FMT == MXP_FMT_MXFP6P || FMT == MXP_FMT_MXFP8P;
    uint32_t m[8], sg[8], lo, hi;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = raw[i] & 0x7FFFFFFFu;
      sg[i] = raw[i] >> 31;
    }
    if constexpr (FMT <= MXP_FMT_MXFP6P) {
      encode_fp6_group<false, PLUS>(raw, m, part, lo, hi, sb, idx);
      if (part < 3u) *reinterpret_cast<u32x2*>(a.elems + blk * 24 + part * 8) = u32x2{lo, hi};
    } else {
      encode_wide_group<false, 8, PLUS>(raw, m, sg, part, lo, hi, sb, idx);
      *reinterpret_cast<u32x2*>(a.elems + blk * 32 + part * 8) = u32x2{lo, hi};
    }
  }
  if (part == 0u) {
    a.scales[blk] = (uint8_t)sb;
    if (FMT != MXP_FMT_MXFP4 && FMT != MXP_FMT_MXFP6 && FMT != MXP_FMT_MXFP8) a.bm_idx[blk] = (uint8_t)idx;
  }
}

// the sum over the workgroup, the same in every lane; `part`: 16 words of shared memory that no lane still reads
__device__ __forceinline__ float block_sum(float s, float* part) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if (waves == 1) return s;
  if ((threadIdx.x & 63) == 0) part[wave] = s;
  __syncthreads();
  s = 0.0f;
  for (int i = 0; i < waves; ++i) s += part[i];
  return s;
}

// (sum(h^2) / K + eps)^-1/2, by an IEEE division and root: once a row
__device__ __forceinline__ float row_scale(const NormArgs& a, float s) { return 1.0f / sqrtf(s / (float)a.K + a.eps); }

template <int FMT>
__device__ __forceinline__ void norm_store(const NormArgs& a, int64_t row, int g, float rs, const float (&v)[8]) {
  float w[8], y[8];
  if (a.w_bf16) load8<true>(a.w, (int64_t)g * 8, w);
  else load8<false>(a.w, (int64_t)g * 8, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i] * rs * w[i];
  convert_store<FMT>(a, row, g, y);
}

// K <= 16 * lanes: the row stays in registers
constexpr int kRowGroups = 2;
template <bool BF16, int FMT>
__global__ void __launch_bounds__(1024) rmsnorm_quantize_kernel(const NormArgs a) {
  __shared__ float part[2][16];
  const int groups = a.K >> 3;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float v[kRowGroups][8], s = 0.0f;
#pragma unroll
    for (int u = 0; u < kRowGroups; ++u) {
      const int g = u * (int)blockDim.x + (int)threadIdx.x;
      if (g < groups) {
        load_sum<BF16>(a, row, g, v[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[u][i] * v[u][i];
      }
    }
    const float rs = row_scale(a, block_sum(s, part[turn]));         // (two rows' sums in turn: one barrier a row)
#pragma unroll
    for (int u = 0; u < kRowGroups; ++u) {
      const int g = u * (int)blockDim.x + (int)threadIdx.x;
      if (g < groups) {
        if (a.h) store8<BF16>(a.h, row * a.ld_h + g * 8, v[u]);
        norm_store<FMT>(a, row, g, rs, v[u]);
      }
    }
  }
}

// longer rows: two passes; h may be x or r itself, so the second pass reads h where it is kept
template <bool BF16, int FMT>
__global__ void __launch_bounds__(1024) rmsnorm_quantize_long_kernel(const NormArgs a) {
  __shared__ float part[2][16];
  const int groups = a.K >> 3;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float s = 0.0f;
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
      float v[8];
      load_sum<BF16>(a, row, g, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i] * v[i];
      if (a.h) store8<BF16>(a.h, row * a.ld_h + g * 8, v);
    }
    const float rs = row_scale(a, block_sum(s, part[turn]));
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
      float v[8];
      if (a.h) load8<BF16>(a.h, row * a.ld_h + g * 8, v);
      else load_sum<BF16>(a, row, g, v);
      norm_store<FMT>(a, row, g, rs, v);
    }
  }
}

template <bool BF16, int FMT>
int norm_launch(const NormArgs& a, hipStream_t s) {
  const int64_t cap = (int64_t)kNumCU * 64;
  const dim3 grid((unsigned)(a.rows < cap ? a.rows : cap));
  const int lanes = (a.K / (8 * kRowGroups) + 63) / 64 * 64;
  if (a.K <= 1024 * 8 * kRowGroups)
    hipLaunchKernelGGL((rmsnorm_quantize_kernel<BF16, FMT>), grid, dim3(lanes < 64 ? 64 : lanes), 0, s, a);
  else
    hipLaunchKernelGGL((rmsnorm_quantize_long_kernel<BF16, FMT>), grid, dim3(1024), 0, s, a);
  return launch_status();
}

}  // namespace

extern "C" int mxp_rmsnorm_quantize(const void* x, const void* residual, int x_dtype, int64_t rows, int64_t K, int64_t ld_x, int64_t ld_residual,
                                    const void* weight, int w_dtype, float eps, void* h, int64_t ld_h, int fmt, uint8_t* elems, uint8_t* scales,
                                    uint8_t* bm_idx, void* stream) {
  using namespace mxp;
  if (fmt < MXP_FMT_MXFP4 || fmt > MXP_FMT_MXFP8P) return MXP_ERR_FORMAT;
  if ((x_dtype != MXP_F32 && x_dtype != MXP_BF16) || (w_dtype != MXP_F32 && w_dtype != MXP_BF16)) return MXP_ERR_DTYPE;
  if (rows < 0 || K < 0 || K % kBlock != 0 || !(eps >= 0.0f && eps < __builtin_inff())) return MXP_ERR_SHAPE;
  if (rows == 0 || K == 0) return MXP_OK;
  if (K > kMaxGemmK) return MXP_ERR_UNSUPPORTED;
  const bool plain = fmt == MXP_FMT_MXFP4 || plain_wide_format(fmt);
  if (!x || !weight || !elems || !scales || (!plain && !bm_idx)) return MXP_ERR_NULL;
  if (ld_x < K || (residual && ld_residual < K) || (h && ld_h < K)) return MXP_ERR_SHAPE;
  const int64_t esz = x_dtype == MXP_BF16 ? 2 : 4;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(h) || !aligned16(elems) || !aligned16(scales) || !aligned16(bm_idx) ||
      ld_x * esz % 16 != 0 || (residual && ld_residual * esz % 16 != 0) || (h && ld_h * esz % 16 != 0))
    return MXP_ERR_ALIGN;
  const NormArgs a{x, residual, weight, h, rows, ld_x, ld_residual, ld_h, (int)K, w_dtype == MXP_BF16, eps, elems, scales, bm_idx};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = x_dtype == MXP_BF16;
#define MXP_NORM(F) case F: return bf ? norm_launch<true, F>(a, s) : norm_launch<false, F>(a, s)
  switch (fmt) {
    MXP_NORM(MXP_FMT_MXFP4);
    MXP_NORM(MXP_FMT_MXFP4P);
    MXP_NORM(MXP_FMT_MXFP4PP);
    MXP_NORM(MXP_FMT_MXFP6);
    MXP_NORM(MXP_FMT_MXFP6P);
    MXP_NORM(MXP_FMT_MXFP8);
    MXP_NORM(MXP_FMT_MXFP8P);
  }
#undef MXP_NORM
  return MXP_ERR_FORMAT;
}
