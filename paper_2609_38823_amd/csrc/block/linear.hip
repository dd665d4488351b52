// Products of few rows with 4-bit weights (e2m1, a power-of-two scale for
// every 32 columns):  y[t, r] = sum_c x[t, c] w[r, c].
//
// A workgroup takes 16, 32 or 64 weight rows and up to 64 rows of x; its eight
// wavefronts take the 128-column steps in turn and their sums are joined in
// LDS in a fixed order.  The operands of a 16-row matrix instruction lie in 16
// rows of memory for every quarter of a wavefront, which the vector cache
// serves a row at a time (measured: 64 cycles a load instead of 16; 37 rows, n
// 8192, k 8192: 58 us), so every wavefront loads whole pieces of rows and
// makes the operands from its own part of LDS (20 us).  A lane's 32 columns
// of a weight row are the first operand of one scaled 16x16x128 instruction
// (8-bit x: no conversion at all), or, converted two values at a time (exact),
// of four bf16 ones; float32 x takes float32 ones.
//
// Bound: few rows by the weights (one row, n 28672, k 8192: 23 us for 125 MB,
// 5.4 TB/s); many rows by the vector cache and LDS, through which every
// workgroup takes all of x (37 rows, n 8192, k 8192: 26 and 17 thousand of the
// kernel's 45 thousand cycles).
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

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int LW = 8;  // wavefronts a workgroup: parts of the columns

// a group's four results of a lane: row t of y, columns col .. + 4
__device__ __forceinline__ void store4(void* y, int y_bf16, size_t o, int col, int n, const f32x4& a) {
  if (y_bf16) {
    uint16_t* p = static_cast<uint16_t*>(y) + o;
    if (col + 4 <= n) {
      store_raw(p, make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3])));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < n) p[i] = f32_to_bf16(a[i]);
    }
  } else {
    float* p = static_cast<float*>(y) + o;
    if (col + 4 <= n) {
      store_raw(p, make_float4(a[0], a[1], a[2], a[3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < n) p[i] = a[i];
    }
  }
}

// add up the wavefronts' accumulators, halves at a time in LDS (a fixed
// order), and store them.  Lane c holds row t0 + 16 j + c of y, columns
// n0 + 16 r + 4 g .. + 4
template <int RT, int TT>
__device__ __forceinline__ void join_store(f32x4 (&acc)[RT][TT], f32x4* part, int wv, int lane, int n0, int t0, int T,
                                           int n, void* y, int y_bf16) {
#pragma unroll
  for (int half = LW / 2; half >= 1; half /= 2) {
    if (wv >= half && wv < 2 * half)
#pragma unroll
      for (int i = 0; i < RT * TT; ++i) part[((wv - half) * RT * TT + i) * 64 + lane] = acc[i / TT][i % TT];
    __syncthreads();
    if (wv < half)
#pragma unroll
      for (int i = 0; i < RT * TT; ++i) acc[i / TT][i % TT] += part[(wv * RT * TT + i) * 64 + lane];
    if (half > 1) __syncthreads();
  }
  if (wv) return;
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      const int t = t0 + j * 16 + (lane & 15), col = n0 + r * 16 + (lane >> 4) * 4;
      if (t < T && col < n) store4(y, y_bf16, (size_t)t * n + col, col, n, acc[r][j]);
    }
}

// The scale bytes of blocks [4 st, 4 st + 4 N) of a row of nb >= 4 N, in one
// load without a branch: what would pass the row's end is read from the row's
// last 4 N bytes, and place_scales, once the bytes are wanted, shifts them
// (behind the end comes 0).
template <int N>
struct Words { uint32_t w[N]; };
template <int N>
__device__ __forceinline__ Words<N> load_scales(const uint8_t* row, int st, int nb) {
  return load_raw<Words<N>>(row + min(4 * st, nb - 4 * N));
}
template <int N>
__device__ __forceinline__ Words<N> place_scales(Words<N> v, int st, int nb) {
  const int off = max(0, 4 * st - max(nb - 4 * N, 0)) * 8;  // (uniform)
  if constexpr (N == 1) {
    v.w[0] >>= off;
  } else {
    const uint64_t w = ((uint64_t)v.w[1] << 32 | v.w[0]) >> off;
    v.w[0] = static_cast<uint32_t>(w);
    v.w[1] = static_cast<uint32_t>(w >> 32);
  }
  return v;
}

// bytes of one wavefront's tiles in LDS (rows padded by 16 bytes: then the 16
// lanes that read a column each touch other banks)
template <bool MX, int TT, int RT, int C, bool FEW>
struct Tile {
  static constexpr int XR = FEW ? 4 : 16 * TT;                  // rows of x
  static constexpr int XB = (MX ? 128 : 256) * C, WB = 64 * C;  // bytes of a row of x, of the weights, in C steps
  static constexpr int XP = XB + 16, WP = WB + 16;
  static constexpr int BYTES = XR * XP + RT * 16 * WP;
  static constexpr int JOIN = (LW / 2) * RT * TT * 1024;
  static constexpr int LDS = LW * BYTES > JOIN ? LW * BYTES : JOIN;
};

// RT groups of 16 weight rows, TT groups of 16 rows of x.  A wavefront takes C
// steps of 128 columns at a time: it has the values of the next C steps in
// flight in registers, in whole pieces of rows as the vector cache serves them
// best, and turns them into operands through its own part of LDS.  FEW: up to
// four rows of x, which stand in all columns (those behind them are not
// stored); then the registers hold another C steps, and memory's latency is
// covered (n 2048, k 4096: 5.0 -> 4.2 us; with more rows, whose LDS traffic
// and loads from cache take the time, it gains nothing).
template <bool MX, int TT, int RT, int C, bool FEW>
__global__ __launch_bounds__(64 * LW) void linear_w4_kernel(const char* __restrict__ x,
                                                            const uint8_t* __restrict__ x_scale, int T, int k,
                                                            const uint8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ scales, int n,
                                                            void* __restrict__ y, int y_bf16) {
  using L = Tile<MX, TT, RT, C, FEW>;
  constexpr int XQ = L::XB / 16, WQ = L::WB / 16;               // 16-byte pieces of a row
  constexpr int NX = (L::XR * XQ + 63) / 64, NW = RT * C;  // and of a lane
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * (16 * RT), t0 = blockIdx.y * (16 * TT);
  const int nb = k / 32, steps = (nb + 3) / 4;
  char* xl = lds + wv * L::BYTES;
  char* wl = xl + L::XR * L::XP;
  const int xr = FEW ? c & 3 : c;  // the row of x in a lane's column (FEW: the four again and again)

  // rows behind the last are the last one again, where a load holds others too;
  // they are not stored
  const uint32_t x_row = (uint32_t)k * (MX ? 1 : 2), w_row = (uint32_t)k / 2;
  const char* xb = x + (size_t)t0 * x_row;
  const uint8_t* wb = codes + (size_t)n0 * w_row;
  uint32_t xo[NX], wo[NW];
#pragma unroll
  for (int i = 0; i < NX; ++i) xo[i] = (uint32_t)min((i * 64 + lane) / XQ, T - 1 - t0) * x_row;
#pragma unroll
  for (int i = 0; i < NW; ++i) wo[i] = (uint32_t)min((i * 64 + lane) / WQ, n - 1 - n0) * w_row;
  const uint32_t xc = (lane % XQ) * 16, wc = (lane % WQ) * 16;  // (64 is a multiple of both)
  const uint8_t* ws_row = scales + (size_t)(n0 + min(lane, min(16 * RT - 1, n - 1 - n0))) * nb;
  const uint8_t* xs_row = MX ? x_scale + (size_t)(t0 + min(lane, min(16 * TT - 1, T - 1 - t0))) * nb : nullptr;

  f32x4 acc[RT][TT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Loads return in order and are counted: there is no branch around any of
  // them.  Pieces behind the end are read again from within and set to 0 on the
  // way into LDS.
  struct Chunk {
    u32x4 x[NX], w[NW];
    Words<C> ws, xs;
  };
  auto fetch_rows = [&](int ch, Chunk& u) {
    const uint32_t wa = min((uint32_t)ch * L::WB + wc, w_row - 16), xa = min((uint32_t)ch * L::XB + xc, x_row - 16);
#pragma unroll
    for (int i = 0; i < NW; ++i) u.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wb + (wo[i] + wa)));
#pragma unroll
    for (int i = 0; i < NX; ++i) u.x[i] = *reinterpret_cast<const u32x4*>(xb + (xo[i] + xa));
  };
  auto fetch = [&](int ch, Chunk& u) {
    fetch_rows(ch, u);
    u.ws = load_scales<C>(ws_row, ch * C, nb);
    if constexpr (MX) u.xs = load_scales<C>(xs_row, ch * C, nb);
  };
  uint32_t sw[RT][C], sx[TT][C];
  auto place = [&](int ch, const Chunk& u) {
    const Words<C> w = place_scales<C>(u.ws, ch * C, nb), v = MX ? place_scales<C>(u.xs, ch * C, nb) : w;
#pragma unroll
    for (int q = 0; q < C; ++q) {
#pragma unroll
      for (int r = 0; r < RT; ++r) sw[r][q] = __shfl(static_cast<int>(w.w[q]), r * 16 + c, 64);
#pragma unroll
      for (int j = 0; j < TT; ++j) sx[j][q] = MX ? __shfl(static_cast<int>(v.w[q]), j * 16 + c, 64) : 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tiles' last reads are behind
    auto store = [&](uint32_t w_in, uint32_t x_in) {
#pragma unroll
      for (int i = 0; i < NW; ++i) *reinterpret_cast<u32x4*>(wl + (i * 64 + lane) / WQ * L::WP + wc) = u.w[i] & w_in;
#pragma unroll
      for (int i = 0; i < NX; ++i) *reinterpret_cast<u32x4*>(xl + (i * 64 + lane) / XQ * L::XP + xc) = u.x[i] & x_in;
    };
    if ((uint32_t)(ch + 1) * L::WB <= w_row) store(~0u, ~0u);  // a whole chunk
    else store((uint32_t)ch * L::WB + wc < w_row ? ~0u : 0u, (uint32_t)ch * L::XB + xc < x_row ? ~0u : 0u);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  auto multiply = [&]() {
#pragma unroll
    for (int q = 0; q < C; ++q) {
      if constexpr (MX) {
        i32x8 B[TT];
#pragma unroll
        for (int j = 0; j < TT; ++j) {
          // the second operand of a lane: bytes 16 g .. + 16 of either half of the
          // step's 128 columns, with the scale of the step's block g
          const char* p = xl + (j * 16 + xr) * L::XP + q * 128 + g * 16;
          const uint4 lo = *reinterpret_cast<const uint4*>(p), hi = *reinterpret_cast<const uint4*>(p + 64);
          B[j] = i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const uint4 w = *reinterpret_cast<const uint4*>(wl + (r * 16 + c) * L::WP + q * 64 + g * 16);
          const i32x8 A = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < TT; ++j)
            acc[r][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                A, B[j], acc[r][j], 4, 0, 0, (int)(sw[r][q] >> (8 * g)), 0, (int)(sx[j][q] >> (8 * g)));
        }
      } else {
#pragma unroll
        for (int m = 0; m < 4; ++m) {  // a block of 32 columns: a lane takes 8 g .. + 8 of it
          uint4 B[TT];
#pragma unroll
          for (int j = 0; j < TT; ++j)
            B[j] = *reinterpret_cast<const uint4*>(xl + (j * 16 + xr) * L::XP + q * 256 + m * 64 + g * 16);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(wl + (r * 16 + c) * L::WP + q * 64 + m * 16 + g * 4);
            const uint32_t byte = (sw[r][q] >> (8 * m)) & 255u;
            const float sc = mx_scale(byte);
            const bf16x2_t a0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0);
            const bf16x2_t a1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1);
            const bf16x2_t a2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2);
            const bf16x2_t a3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3);
            const bf16x8 A = {a0[0], a0[1], a1[0], a1[1], a2[0], a2[1], a3[0], a3[1]};
#pragma unroll
            for (int j = 0; j < TT; ++j)
              acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8, B[j]), acc[r][j], 0, 0,
                                                                  0);
          }
        }
      }
    }
  };
  const int chunks = (steps + C - 1) / C;
  const int mine = wv < chunks ? (chunks - 1 - wv) / LW + 1 : 0;  // of this wavefront: wv, wv + LW, ...
  if (mine == 1) {
    Chunk u;
    if (nb >= 4 * C) {
      fetch(wv, u);
    } else {  // a single chunk, not a whole one
      fetch_rows(wv, u);
#pragma unroll
      for (int q = 0; q < C; ++q) u.ws.w[q] = u.xs.w[q] = 0;
#pragma unroll
      for (int b = 0; b < 4 * C; ++b)
        if (b < nb) {
          u.ws.w[b / 4] |= (uint32_t)ws_row[b] << (8 * (b % 4));
          if constexpr (MX) u.xs.w[b / 4] |= (uint32_t)xs_row[b] << (8 * (b % 4));
        }
    }
    place(wv, u);
    multiply();
  } else if (mine > 1 && !FEW) {
    Chunk u;
    fetch(wv, u);
    for (int ch = wv; ch < chunks; ch += LW) {
      place(ch, u);
      if (ch + LW < chunks) fetch(ch + LW, u);
      multiply();
    }
  } else if (mine > 1) {  // two chunks ahead
    Chunk even, odd;
    int ch = wv, left = mine;
    fetch(ch, even);
    fetch(ch + LW, odd);
    for (; left > 3; left -= 2, ch += 2 * LW) {
      place(ch, even);
      fetch(ch + 2 * LW, even);
      multiply();
      place(ch + LW, odd);
      fetch(ch + 3 * LW, odd);
      multiply();
    }
    place(ch, even);
    if (left == 3) {
      fetch(ch + 2 * LW, even);
      multiply();
      place(ch + LW, odd);
      multiply();
      place(ch + 2 * LW, even);
      multiply();
    } else {
      multiply();
      place(ch + LW, odd);
      multiply();
    }
  }
  __syncthreads();  // the tiles' LDS becomes the join's
  join_store<RT, TT>(acc, reinterpret_cast<f32x4*>(lds), wv, lane, n0, t0, T, n, y, y_bf16);
}

// float32 rows: operands straight from memory (the float32 matrix instructions
// bound it, not the loads)
template <int TT>
__global__ __launch_bounds__(64 * LW) void linear_w4_f32_kernel(const float* __restrict__ x, int T, int k,
                                                                const uint8_t* __restrict__ codes,
                                                                const uint8_t* __restrict__ scales, int n,
                                                                void* __restrict__ y, int y_bf16) {
  __shared__ f32x4 part[(LW / 2) * TT * 64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, t0 = blockIdx.y * (16 * TT);
  const int nb = k / 32, steps = (nb + 3) / 4;
  const int wr = min(n0 + c, n - 1);
  const uint8_t* wc = codes + (size_t)wr * (k / 2) + g * 16;
  const uint8_t* ws = scales + (size_t)wr * nb + g;
  f32x4 acc[1][TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) acc[0][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int st = wv; st < steps; st += LW) {
    const int b = st * 4 + g;  // this lane's block of 32 columns
    const bool in = b < nb;
    const uint4 w = in ? load_stream(reinterpret_cast<const uint4*>(wc + (size_t)st * 64)) : make_uint4(0, 0, 0, 0);
    const uint32_t byte = in ? ws[st * 4] : 127u;
    const uint32_t wd[4] = {w.x, w.y, w.z, w.w};
    const float sc = mx_scale(byte);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 0);
      const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 1);
      const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 2);
      const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wd[m], sc, 3);
      const float A[8] = {a0[0], a0[1], a1[0], a1[1], a2[0], a2[1], a3[0], a3[1]};
#pragma unroll
      for (int j = 0; j < TT; ++j) {
        const float* xp = x + (size_t)min(t0 + j * 16 + c, T - 1) * k + (size_t)b * 32 + m * 8;
        float4 p = make_float4(0.f, 0.f, 0.f, 0.f), h = p;
        if (in) p = *reinterpret_cast<const float4*>(xp), h = *reinterpret_cast<const float4*>(xp + 4);
        const float B[8] = {p.x, p.y, p.z, p.w, h.x, h.y, h.z, h.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[e], B[e], acc[0][j], 0, 0, 0);
      }
    }
  }
  join_store<1, TT>(acc, part, wv, lane, n0, t0, T, n, y, y_bf16);
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
  const int tt = T <= 16 ? 1 : T <= 32 ? 2 : T <= 48 ? 3 : 4;
  // Groups of 16 weight rows a workgroup.  Each workgroup reads all of x again
  // and its LDS leaves room for one on a compute unit (8-bit x of up to 16 rows:
  // for three), so as many groups as make it one workgroup for each of the 256.
  // 1 / 2 / 4 groups, us: bf16, n 2048, k 4096, 16 rows 5.1 / 5.5 / 7.5; n
  // 5120, k 2048, 37 rows 10.7 / 6.9 / 10.1; n 16384, k 4096, 37 rows 34 / 23 /
  // 18; 8-bit, 16 rows (1 / 2): n 5120, k 2048 4.4 / 4.2; n 8192, k 8192 12.4 /
  // 10.5.  Up to four rows of x leave room for several and are read again for
  // little: 8-bit one group (one row, n 28672, k 8192: 23.1 / 27.1), bf16 two
  // where they still fill the chip (26.5 / 24.9 / 28.6; n 5120, k 2048 4.1 /
  // 4.1 / 5.4).
  const bool few = T <= 4;
  const int groups = (n + 15) / 16;
  int rt = groups <= 256 ? 1 : groups <= 512 ? 2 : 4;
  if (x_kind == kMx && tt == 1) rt = groups < 512 ? 1 : 2;
  if (x_kind == 1 && tt == 4) rt = std::min(rt, 2);  // (four groups: more LDS than there is)
  if (few) rt = x_kind == kMx || groups <= 512 ? 1 : 2;
#define RUN(MX, TT, RT, C, FEW)                                                                                \
  linear_w4_kernel<MX, TT, RT, C, FEW>                                                                         \
      <<<dim3((n + 16 * RT - 1) / (16 * RT), (T + 16 * TT - 1) / (16 * TT)), 64 * LW, Tile<MX, TT, RT, C, FEW>::LDS, \
         s>>>(static_cast<const char*>(x), x_scale, T, k, codes, scales, n, y, y_bf16)
#define ROWS(MX, TT, C, MOST)                                    \
  do {                                                           \
    if (rt == 1) RUN(MX, TT, 1, C, false);                       \
    else if (rt == 2) RUN(MX, TT, 2, C, false);                  \
    else if constexpr (MOST == 4) RUN(MX, TT, 4, C, false);      \
  } while (0)
  if (x_kind == kMx) {
    if (few) RUN(true, 1, 1, 2, true);
    else if (tt == 1) ROWS(true, 1, 2, 2);
    else if (tt == 2) ROWS(true, 2, 2, 4);
    else if (tt == 3) ROWS(true, 3, 1, 4);
    else ROWS(true, 4, 1, 4);
  } else if (x_kind == 1) {
    if (few && rt == 1) RUN(false, 1, 1, 2, true);
    else if (few) RUN(false, 1, 2, 2, true);
    else if (tt == 1) ROWS(false, 1, 2, 4);
    else if (tt == 2) ROWS(false, 2, 1, 4);
    else if (tt == 3) ROWS(false, 3, 1, 4);
    else ROWS(false, 4, 1, 2);
  } else {
#define F32(TT)                                                                                              \
  linear_w4_f32_kernel<TT><<<dim3((n + 15) / 16, (T + 16 * TT - 1) / (16 * TT)), 64 * LW, 0, s>>>(           \
      static_cast<const float*>(x), T, k, codes, scales, n, y, y_bf16)
    if (tt == 1) F32(1);
    else if (tt == 2) F32(2);
    else if (tt == 3) F32(3);
    else F32(4);
#undef F32
  }
#undef ROWS
#undef RUN
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
