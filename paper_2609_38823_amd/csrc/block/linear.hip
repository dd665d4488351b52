// Products of few rows with 4-bit weights (e2m1, a power-of-two scale for
// every 32 columns):  y[t, r] = sum_c x[t, c] w[r, c].
//
// A workgroup takes 16 weight rows and up to 64 rows of x; its four
// wavefronts take the 128-column steps in turn and their sums are joined in
// LDS in a fixed order.  A lane reads its 32 columns of a weight row as one
// 16-byte load: the first operand of one scaled 16x16x128 matrix instruction
// (8-bit x: no conversion at all), or, converted two values at a time (exact),
// of four bf16 ones or 32 float32 ones.  The weights are read once for every
// 64 rows, which is what bounds it.
//
// Rounding: the scaled instruction aligns the exact products of eight
// neighbouring columns to the largest and keeps 13 bits below its exponent
// before it adds in float32 (measured: next to 448 * 6, 2^-3 is kept and 2^-4
// is not; columns further away are not touched).  It is taken all the same:
// against the 2^-4 that a value of x has already lost in becoming e4m3, and
// the half step of 2^-8 of a bf16 result, the loss is nothing (root mean
// square 2^-17 of sum |x w| on normal data), and it saves every conversion.
#include "block.hpp"

#include <algorithm>

namespace decomoe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int LW = 4;  // wavefronts a workgroup: parts of the columns

template <int KIND, int TT>
__global__ __launch_bounds__(64 * LW) void linear_w4_kernel(const void* __restrict__ x,
                                                            const uint8_t* __restrict__ x_scale, int T, int k,
                                                            const uint8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ scales, int n,
                                                            void* __restrict__ y, int y_bf16) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, t0 = blockIdx.y * (16 * TT);
  const int nb = k / 32, steps = (nb + 3) / 4;
  const int wr = min(n0 + c, n - 1);  // a row behind the last is not stored
  const uint8_t* wc = codes + (size_t)wr * (k / 2) + g * 16;
  const uint8_t* ws = scales + (size_t)wr * nb + g;
  size_t xr[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) xr[j] = (size_t)min(t0 + j * 16 + c, T - 1);
  f32x4 acc[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int st = wv; st < steps; st += LW) {
    const int b = st * 4 + g;  // this lane's block of 32 columns
    const bool in = b < nb;
    uint4 w = make_uint4(0, 0, 0, 0);
    uint32_t sw = 127;
    if (in) {
      w = load_stream(reinterpret_cast<const uint4*>(wc + (size_t)st * 64));
      sw = ws[st * 4];
    }
    if constexpr (KIND == kMx) {
      const i32x8 A = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
      // the second operand of a lane: bytes 16 g .. + 16 of either half of the
      // step's 128 columns, with the scale of the step's block g
      const bool lo = st * 4 + g / 2 < nb, hi = st * 4 + 2 + g / 2 < nb;
#pragma unroll
      for (int j = 0; j < TT; ++j) {
        const uint8_t* xp = static_cast<const uint8_t*>(x) + xr[j] * k + (size_t)st * 128 + g * 16;
        uint4 p = make_uint4(0, 0, 0, 0), q = p;
        if (lo) p = *reinterpret_cast<const uint4*>(xp);
        if (hi) q = *reinterpret_cast<const uint4*>(xp + 64);
        const uint32_t sx = in ? x_scale[xr[j] * nb + b] : 127u;
        const i32x8 B = {(int)p.x, (int)p.y, (int)p.z, (int)p.w, (int)q.x, (int)q.y, (int)q.z, (int)q.w};
        acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc[j], 4, 0, 0, (int)sw, 0, (int)sx);
      }
    } else {
      const uint32_t wd[4] = {w.x, w.y, w.z, w.w};
      const float sc = sw == 255u ? __uint_as_float(0x7fc00000u) : mx_scale(sw);
      if constexpr (KIND == 1) {
        bf16x8 A[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const bf16x2_t a0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd[m], sc, 0);
          const bf16x2_t a1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd[m], sc, 1);
          const bf16x2_t a2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd[m], sc, 2);
          const bf16x2_t a3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wd[m], sc, 3);
          A[m] = bf16x8{a0[0], a0[1], a1[0], a1[1], a2[0], a2[1], a3[0], a3[1]};
        }
#pragma unroll
        for (int j = 0; j < TT; ++j) {
          const uint16_t* xp = static_cast<const uint16_t*>(x) + xr[j] * k + (size_t)b * 32;
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (in) q = *reinterpret_cast<const uint4*>(xp + m * 8);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[m], __builtin_bit_cast(bf16x8, q), acc[j], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 0);
          const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 1);
          const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 2);
          const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 3);
          const float A[8] = {a0[0], a0[1], a1[0], a1[1], a2[0], a2[1], a3[0], a3[1]};
#pragma unroll
          for (int j = 0; j < TT; ++j) {
            const float* xp = static_cast<const float*>(x) + xr[j] * k + (size_t)b * 32 + m * 8;
            float4 p = make_float4(0.f, 0.f, 0.f, 0.f), q = p;
            if (in) p = *reinterpret_cast<const float4*>(xp), q = *reinterpret_cast<const float4*>(xp + 4);
            const float B[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[e], B[e], acc[j], 0, 0, 0);
          }
        }
      }
    }
  }

  // join the wavefronts' sums: lane c holds row t0 + 16 j + c of y, columns
  // n0 + 4 g .. + 4
  __shared__ f32x4 part[LW - 1][TT][64];
  if (wv)
#pragma unroll
    for (int j = 0; j < TT; ++j) part[wv - 1][j][lane] = acc[j];
  __syncthreads();
  if (wv) return;
#pragma unroll
  for (int j = 0; j < TT; ++j) {
#pragma unroll
    for (int p = 0; p < LW - 1; ++p) acc[j] += part[p][j][lane];
    const int t = t0 + j * 16 + c;
    if (t >= T) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = n0 + g * 4 + i;
      if (r >= n) break;
      const size_t o = (size_t)t * n + r;
      if (y_bf16) static_cast<uint16_t*>(y)[o] = f32_to_bf16(acc[j][i]);
      else static_cast<float*>(y)[o] = acc[j][i];
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(256) void quantize_w4_kernel(const void* __restrict__ w, size_t blocks,
                                                          uint8_t* __restrict__ codes,
                                                          uint8_t* __restrict__ scales) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < blocks * 4; i += (size_t)gridDim.x * 256) {
    float v[8];  // a lane's eight of a block of 32; blocks * 4 is a multiple of 4: whole groups of lanes
    load8<BF16>(static_cast<const char*>(w) + i * 8 * (BF16 ? 2 : 4), 0, 8, v);
    const uint32_t byte = mx4_byte(block_most(v));
    const float inv = mx_inverse(byte);
    uint32_t out = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // the values lie between 0, 0.5, 1, 1.5, 2, 3, 4, 6: ties go to the even code
      const float m = fabsf(v[e] * inv);
      const uint32_t code = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) +
                            (m > 5.f);
      out |= (code | (__float_as_uint(v[e]) >> 31 << 3)) << (4 * e);
    }
    reinterpret_cast<uint32_t*>(codes)[i] = out;
    if ((i & 3) == 0) scales[i >> 2] = static_cast<uint8_t>(byte);
  }
}

}  // namespace

hipError_t launch_linear_w4(const void* x, int x_kind, const uint8_t* x_scale, int T, int k, const uint8_t* codes,
                            const uint8_t* scales, int n, void* y, bool y_bf16, hipStream_t s) {
  const unsigned nx = (n + 15) / 16;
#define LINEAR(TT)                                                                                                \
  do {                                                                                                            \
    const dim3 g(nx, (T + 16 * TT - 1) / (16 * TT));                                                              \
    if (x_kind == kMx)                                                                                            \
      linear_w4_kernel<kMx, TT><<<g, 64 * LW, 0, s>>>(x, x_scale, T, k, codes, scales, n, y, y_bf16);             \
    else if (x_kind == 1)                                                                                         \
      linear_w4_kernel<1, TT><<<g, 64 * LW, 0, s>>>(x, x_scale, T, k, codes, scales, n, y, y_bf16);               \
    else                                                                                                          \
      linear_w4_kernel<0, TT><<<g, 64 * LW, 0, s>>>(x, x_scale, T, k, codes, scales, n, y, y_bf16);               \
  } while (0)
  if (T <= 16) LINEAR(1);
  else if (T <= 32) LINEAR(2);
  else LINEAR(4);
#undef LINEAR
  return hipGetLastError();
}

hipError_t launch_quantize_w4(const void* w, bool bf16, int n, int k, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const size_t blocks = (size_t)n * (k / 32);
  const unsigned grid = (unsigned)std::min<size_t>((blocks * 4 + 255) / 256, 16384);
  if (bf16) quantize_w4_kernel<true><<<grid, 256, 0, s>>>(w, blocks, codes, scales);
  else quantize_w4_kernel<false><<<grid, 256, 0, s>>>(w, blocks, codes, scales);
  return hipGetLastError();
}

}  // namespace decomoe
