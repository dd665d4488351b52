// RMS norm with the residual's addition; 16-bit or 8-bit output.
//
//   h = x + r,  y = h * rsqrt(mean(h^2) + eps) * w
//
// One pass: a row is read once into registers (8 values a lane and chunk),
// summed, and written in every form that was asked for.  Four neighbouring
// lanes hold a microscaling block of 32 values, so its maximum is two lane
// exchanges.  Sums have a fixed order.
//
// Bound: memory for many rows (4096 rows of 2048 with residual, sum, rows and
// 8-bit rows: a call 13.8 us for 76 MB, 5.5 TB/s - part of it from the
// memory-side cache), latency for few (one row: the kernel 2.6 us).
#include "block.hpp"

namespace decomoe {
namespace {

// TPR threads a row (64: one wavefront), CH chunks of 8 values a thread
template <bool BF16, int TPR, int CH>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_kernel(
    const void* x, const void* residual, const float* __restrict__ weight, int T, int d, float eps, void* h_out,
    void* y, uint8_t* __restrict__ q, uint8_t* __restrict__ q_scale) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1, WPR = TPR / 64, ES = BF16 ? 2 : 4;
  const int tid = threadIdx.x, i = tid % TPR;
  const int t = blockIdx.x * RPB + tid / TPR;
  const bool row = t < T;  // (uniform in a wavefront; workgroups of one row have none without)
  const size_t base = (size_t)(row ? t : T - 1) * d;
  const char* xr = static_cast<const char*>(x) + base * ES;
  const char* rr = residual ? static_cast<const char*>(residual) + base * ES : nullptr;
  float h[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) load8<BF16>(xr, (c * TPR + i) * 8, d, h[c]);
  if (rr) {
    float r[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) load8<BF16>(rr, (c * TPR + i) * 8, d, r[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] += r[c][e];
  }
  // eight squares at a time in float32, the row in 64 bits: one factor for the
  // whole row, so that its error would move every value to the same side
  __shared__ double part[WPR];
  auto row_sum = [&](double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    if constexpr (WPR > 1) {
      if ((tid & 63) == 0) part[tid >> 6] = v;
      __syncthreads();
      v = 0.0;
#pragma unroll
      for (int w = 0; w < WPR; ++w) v += part[w];
    }
    return v;
  };
  double sum = 0.0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float eight = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) eight = fmaf(h[c][e], h[c][e], eight);
    sum += eight;
  }
  sum = row_sum(sum);
  // squares that float32 does not hold (values from 2^60 on, or a whole row
  // below 2^-50): the row again in 64 bits (the branch is the row's)
  if (!(sum > 1e-30 && sum < 1e36)) {
    sum = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma((double)h[c][e], (double)h[c][e], sum);
    if constexpr (WPR > 1) __syncthreads();  // the first sums have been read
    sum = row_sum(sum);
  }
  if (!row) return;
  char* hr = h_out ? static_cast<char*>(h_out) + base * ES : nullptr;
  char* yr = y ? static_cast<char*>(y) + base * ES : nullptr;
  double m = sum / static_cast<double>(d) + eps;
  // a mean at float32's ends is brought to its middle by 2^-132 or 2^200, and
  // the values (h_out first) by the root of that, so that the factor is an
  // ordinary number
  if (!(m > 1e-30 && m < 1e36)) {
    const float pre = m > 1.0 ? 0x1p-66f : 0x1p100f;
    m *= static_cast<double>(pre) * static_cast<double>(pre);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (hr) store8<BF16>(hr, (c * TPR + i) * 8, d, h[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] *= pre;
    }
    hr = nullptr;
  }
  // 1 / sqrt(m): the float32 root and one step of Newton's iteration
  float f = rsqrtf(static_cast<float>(m));
  if (m > 0.0 && m < 3e38) f = static_cast<float>(f * (1.5 - 0.5 * m * f * f));
  const int nb = (d + 31) / 32;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * TPR + i) * 8;
    if (hr) store8<BF16>(hr, at, d, h[c]);
    float w[8];
    if (weight) {
      load8<false>(weight, at, d, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * f * w[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * f;
    }
    if (yr) store8<BF16>(yr, at, d, h[c]);
    if (q) {
      // a lane behind the row's end holds zeros, or 0 * infinity of a row that
      // is not finite: it must not reach the block's maximum
      if (at + 8 > d)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e >= d) h[c][e] = 0.f;
      const uint32_t byte = mx8_byte(block_most(h[c]));
      const uint2 v = to_e4m3x8(h[c], mx_inverse(byte));
      if (at + 8 <= d) {
        store_raw(q + base + at, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < d) q[base + at + e] = static_cast<uint8_t>((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
      }
      if (at < d && (i & 3) == 0) q_scale[(size_t)t * nb + (at >> 5)] = static_cast<uint8_t>(byte);
    }
  }
}

}  // namespace

hipError_t launch_rms_norm(const void* x, bool bf16, const void* residual, const float* weight, int T, int d,
                           float eps, void* h_out, void* y, void* q, uint8_t* q_scale, hipStream_t s) {
#define NORM(TPR, CH)                                                                                            \
  do {                                                                                                           \
    const unsigned blocks = TPR < 256 ? (T + 256 / TPR - 1) / (256 / TPR) : T;                                   \
    if (bf16)                                                                                                    \
      rms_norm_kernel<true, TPR, CH><<<blocks, TPR < 256 ? 256 : TPR, 0, s>>>(                                   \
          x, residual, weight, T, d, eps, h_out, y, static_cast<uint8_t*>(q), q_scale);                          \
    else                                                                                                         \
      rms_norm_kernel<false, TPR, CH><<<blocks, TPR < 256 ? 256 : TPR, 0, s>>>(                                  \
          x, residual, weight, T, d, eps, h_out, y, static_cast<uint8_t*>(q), q_scale);                          \
  } while (0)
  // a wavefront, or a workgroup of 256, a row; few long rows take more threads
  // (64 rows of 8192: 256 / 1024 threads 5.9 / 4.1 us, 512 rows 10.3 / 9.2; of
  // 4096, 64 rows 4.0 / 4.0, 512 rows 6.2 / 7.0)
  if (d <= 512) NORM(64, 1);
  else if (d <= 2048) NORM(256, 1);
  else if (d > 4096 && d <= 8192 && T <= 512) NORM(1024, 1);
  else if (d <= 4096) NORM(256, 2);
  else if (d <= 8192) NORM(256, 4);
  else NORM(1024, 4);
#undef NORM
  return hipGetLastError();
}

}  // namespace decomoe
