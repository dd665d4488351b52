// Device helpers and launcher declarations of the attention half of a block.
#pragma once

#include "../common.hpp"

namespace decomoe {

constexpr int kMx = 2;  // BLK_MX8: e4m3 values with one e8m0 scale for every 32

// ---- unaligned 4-, 8-, 12- and 16-byte accesses -----------------------------
// gfx950 takes vector loads and stores at any address, so rows whose length
// is no multiple of 16 bytes use the same instructions as aligned ones
template <typename V>
__device__ __forceinline__ V load_raw(const void* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <typename V>
__device__ __forceinline__ void store_raw(void* p, const V& v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// ---- rows of bf16 or float32 values as float32 -------------------------------
// values [i, i + 8) of a row, zeros from n on
template <bool BF16>
__device__ __forceinline__ void load8(const void* row, int i, int n, float (&v)[8]) {
  if constexpr (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(row) + i;
    if (i + 8 <= n) {
      const uint4 q = load_raw<uint4>(p);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = i + e < n ? bf16_to_f32(p[e]) : 0.f;
    }
  } else {
    const float* p = static_cast<const float*>(row) + i;
    if (i + 8 <= n) {
      const float4 a = load_raw<float4>(p), b = load_raw<float4>(p + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
      v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = i + e < n ? p[e] : 0.f;
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* row, int i, int n, const float (&v)[8]) {
  if constexpr (BF16) {
    uint16_t* p = static_cast<uint16_t*>(row) + i;
    if (i + 8 <= n) {
      store_raw(p, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                              pack_bf16x2(v[6], v[7])));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < n) p[e] = f32_to_bf16(v[e]);
    }
  } else {
    float* p = static_cast<float*>(row) + i;
    if (i + 8 <= n) {
      store_raw(p, make_float4(v[0], v[1], v[2], v[3]));
      store_raw(p + 4, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < n) p[e] = v[e];
    }
  }
}

// ---- microscaling -------------------------------------------------------------
// The scale byte E + 127 of a block whose largest |v| has the bits `most`
// (integer maximum of the absolute values' bits: NaN and infinity win): the
// smallest E >= -127 with max |v| <= 1.75 * 2^(8 + E) (448, e4m3) or
// 1.5 * 2^(2 + E) (6, e2m1); 255 where the block is not finite.
template <int TOP, uint32_t MANT>
__device__ __forceinline__ uint32_t mx_byte(uint32_t most) {
  if (most >= 0x7f800000u) return 255u;
  const int b = static_cast<int>(most >> 23) - TOP + ((most & 0x7fffffu) > MANT ? 1 : 0);
  return b < 0 ? 0u : static_cast<uint32_t>(b);
}
__device__ __forceinline__ uint32_t mx8_byte(uint32_t most) { return mx_byte<8, 0x600000u>(most); }
__device__ __forceinline__ uint32_t mx4_byte(uint32_t most) { return mx_byte<2, 0x400000u>(most); }
// 2^-E (a block that is not finite: NaN, so that its values come out as NaN)
__device__ __forceinline__ float mx_inverse(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((254u - byte) << 23);
}
// 2^E as the float32 operand of the scaled conversions, which use its exponent
// field alone: byte 0 is 2^-127 (measured: 1 becomes 5.9e-39), byte 255 makes
// NaNs of all values
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// eight values as e4m3 bytes, in order (|v * inv| <= 448: nothing saturates)
__device__ __forceinline__ uint2 to_e4m3x8(const float (&v)[8], float inv) {
  uint2 r;
  r.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
  r.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, r.x, true);
  r.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, 0, false);
  r.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, r.y, true);
  return r;
}
// the largest |v| bits of 32 consecutive values that four neighbouring lanes hold
__device__ __forceinline__ uint32_t block_most(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[e]));
  m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1, 64)));
  return max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2, 64)));
}

// ---- launchers ------------------------------------------------------------------
hipError_t launch_rms_norm(const void* x, bool bf16, const void* residual, const float* weight, int T, int d,
                           float eps, void* h_out, void* y, void* q, uint8_t* q_scale, hipStream_t s);
hipError_t launch_kv_extend(const int32_t* len_in, const int32_t* add, int n_seq, int page_size, int max_pages,
                            int n_pages, int rows_max, const int32_t* n_free_in, int32_t* block_table,
                            int32_t* free_pages, int32_t* len_out, int32_t* n_free_out, int32_t* row_offsets,
                            int32_t* slot_map, int32_t* positions, int32_t* accepted, int32_t* status,
                            hipStream_t s);
hipError_t launch_qkv_cache(const void* qkv, bool bf16, int T, int n_q, int n_kv, int D, const float* q_norm,
                            const float* k_norm, float eps, const int32_t* positions, const float* inv_freq, int rot,
                            const int32_t* slot_map, bool mx, int n_pages, int page_size, void* q_out, void* k_cache,
                            void* v_cache, uint8_t* k_scale, uint8_t* v_scale, hipStream_t s);
bool attn_sizes_ok(int n_seq, int n_q, int n_kv, int D, int max_keys);
size_t attn_ws_bytes(int n_seq, int n_q, int n_kv, int D, int max_keys);
// kind: MOE_F32, MOE_BF16 or kMx of the cache (kMx: bf16 q)
hipError_t launch_attn_decode(const void* q, int kind, int n_seq, int n_q, int n_kv, int D, const void* k_cache,
                              const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int n_pages,
                              int page_size, const int32_t* block_table, int max_pages, const int32_t* lens,
                              float scale, void* out, void* ws, hipStream_t s);
// x_kind: MOE_F32, MOE_BF16 or kMx
hipError_t launch_linear_w4(const void* x, int x_kind, const uint8_t* x_scale, int T, int k, const uint8_t* codes,
                            const uint8_t* scales, int n, void* y, bool y_bf16, hipStream_t s);
hipError_t launch_quantize_w4(const void* w, bool bf16, int n, int k, uint8_t* codes, uint8_t* scales, hipStream_t s);

}  // namespace decomoe
