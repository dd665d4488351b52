// Head norm, rotation and the write into the paged cache.
//
//   v <- v / sqrt(mean(v^2) + eps) * w               query and key heads
//   (v_i, v_{i+r}) <- (v_i cos - v_{i+r} sin, v_{i+r} cos + v_i sin),
//       i < r = rot / 2, angle = position * inv_freq_i
//
// A head is GL lanes of 8 values.  A lane keeps its column over all the heads
// that it takes of a row, so the angles - formed in 64 bits, reduced to a
// fraction of a turn there, then float32 - are computed once a row and lane.
// The partner values of the rotation are read a second time (from cache)
// rather than exchanged.
//
// Bound: memory, and the few wavefronts of a short step by latency (64 rows of
// 32 + 4 + 4 heads of 128: the kernel 4.7 us; 8192 rows: 34, a call 40 us for 168
// MB, 4.2 TB/s, of which 35 are left without norm and rotation).
#include "block.hpp"

#include <algorithm>

namespace decomoe {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct QkvArgs {
  const void* qkv;
  const float *q_norm, *k_norm;
  const int32_t* positions;
  const float* inv_freq;
  const int32_t* slot_map;
  void *q_out, *k_cache, *v_cache;
  uint8_t *k_scale, *v_scale;
  int T, n_q, n_kv, D, rot, n_pages, page, steps;  // steps: of one wavefront
  float eps;
};

template <bool BF16, bool MX, int GL>
__global__ __launch_bounds__(64) void qkv_cache_kernel(const QkvArgs a) {
  constexpr int HPW = 64 / GL, ES = BF16 ? 2 : 4, NV = ES / 2;  // NV: 16-byte pieces of 8 values
  const int lane = threadIdx.x, l = lane % GL, D = a.D, at = l * 8;
  const int t = blockIdx.x, n_all = a.n_q + 2 * a.n_kv, half = a.rot / 2;
  const bool on = at < D;  // (lanes beyond the head's length)
  const int slot = a.slot_map[t];
  const uint32_t pg = (uint32_t)slot / (uint32_t)a.page, off = (uint32_t)slot % (uint32_t)a.page;
  const bool kept = slot >= 0 && pg < (uint32_t)a.n_pages;

  // this lane's rotation: partner column, cosines, signed sines
  const bool turned = at < a.rot;
  const int pair = at < half ? at + half : at - half;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) cs[e] = 1.f, sn[e] = 0.f;
  if (turned) {
    const double p = static_cast<double>(a.positions[t]);
    const int j = at < half ? at : at - half;
    float freq[8];
    load8<false>(a.inv_freq, j, half, freq);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      double u = p * static_cast<double>(freq[e]) * 0.15915494309189533577;  // in turns
      u -= rint(u);
      sincospif(2.f * static_cast<float>(u), &sn[e], &cs[e]);
      if (at < half) sn[e] = -sn[e];
    }
  }

  // steps of HPW heads: the queries', the keys', the values'.  The next step's
  // values are loaded before a step is computed; a lane without a head reads
  // another one's.
  const int n_sq = (a.n_q + HPW - 1) / HPW, n_sk = (a.n_kv + HPW - 1) / HPW;
  const int s_end = min(n_sq + 2 * n_sk, ((int)blockIdx.y + 1) * a.steps);
  const char* row = static_cast<const char*>(a.qkv) + (size_t)t * n_all * D * ES;
  auto kind_of = [&](int st) { return st < n_sq ? 0 : st < n_sq + n_sk ? 1 : 2; };  // (uniform)
  auto head_of = [&](int st) {
    return (st < n_sq ? st : st < n_sq + n_sk ? st - n_sq : st - n_sq - n_sk) * HPW + lane / GL;
  };
  const int in = min(at, D - 8) * ES, in2 = turned ? pair * ES : in;
  auto fetch = [&](int st, u32x4 (&x)[2 * NV]) {
    const int kind = kind_of(st), n = kind == 0 ? a.n_q : a.n_kv;
    const char* src = row + (size_t)((kind == 0 ? 0 : kind == 1 ? a.n_q : a.n_q + a.n_kv) + min(head_of(st), n - 1)) * D * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = *reinterpret_cast<const u32x4*>(src + in + 16 * i);
      x[NV + i] = *reinterpret_cast<const u32x4*>(src + in2 + 16 * i);
    }
  };
  auto floats = [&](const u32x4* x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = BF16 ? __uint_as_float(e & 1 ? x[0][e / 2] & 0xffff0000u : x[0][e / 2] << 16)
                  : __uint_as_float(x[e / 4][e % 4]);
  };
  int have = -1;
  float c[8], d[8];  // v <- f (v c + u d): cosines and sines with the norm's weights
  u32x4 next[2 * NV];
  const int s0 = blockIdx.y * a.steps;
  fetch(s0, next);
  for (int st = s0; st < s_end; ++st) {
    u32x4 now[2 * NV];
#pragma unroll
    for (int i = 0; i < 2 * NV; ++i) now[i] = next[i];
    fetch(min(st + 1, s_end - 1), next);
    const int kind = kind_of(st), h = head_of(st);
    const bool live = on && h < (kind == 0 ? a.n_q : a.n_kv);
    float v[8], u[8];
    floats(now, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = on ? v[e] : 0.f;
    if (kind < 2) {
      const float* weight = kind ? a.k_norm : a.q_norm;
      if (have != kind) {
        have = kind;
        float w[8], x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = x[e] = 1.f;
        if (weight && on) {
          load8<false>(weight, at, D, w);
          if (turned) load8<false>(weight, pair, D, x);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = w[e] * cs[e], d[e] = x[e] * sn[e];
      }
      float f = 1.f;
      if (weight) {
        auto mean = [&](float pre) {  // of the values times a power of two
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = fmaf(v[e] * pre, v[e] * pre, sum);
#pragma unroll
          for (int o = GL / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
          return sum / static_cast<float>(D) + a.eps * pre * pre;
        };
        float m = mean(1.f);
        // squares at float32's ends: the head's values in the middle of its range.
        // The power of two goes into this step's cosines and sines, which the next
        // one forms again: values scaled themselves would outlive the branch, and
        // their registers leave a SIMD five wavefronts instead of six (8192 rows:
        // 43 us a call, so 40, without any of it 39)
        if (__builtin_expect(__ballot(!(m > 1e-30f && m < 1e36f)) != 0, 0)) {
          const float pre = m >= 1e36f ? 0x1p-80f : m <= 1e-30f ? 0x1p100f : 1.f;
          m = mean(pre);
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] *= pre, d[e] *= pre;
          have = -1;
        }
        f = rsqrtf(m);
      }
      floats(now + NV, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = turned ? u[e] : 0.f;  // (an infinity is not to meet the sine's 0)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], c[e], u[e] * d[e]) * f;
    }
    if (kind == 0) {
      if (live) store8<BF16>(static_cast<char*>(a.q_out) + ((size_t)t * a.n_q + h) * D * ES, at, D, v);
      continue;
    }
    const size_t r = ((size_t)pg * a.n_kv + h) * a.page + off;
    char* cache = static_cast<char*>(kind == 1 ? a.k_cache : a.v_cache);
    if constexpr (MX) {
      const uint32_t byte = mx8_byte(block_most(v));
      if (kept && live) {
        store_raw(cache + r * D + at, to_e4m3x8(v, mx_inverse(byte)));
        if ((l & 3) == 0) (kind == 1 ? a.k_scale : a.v_scale)[r * (D / 32) + l / 4] = static_cast<uint8_t>(byte);
      }
    } else {
      if (kept && live) store8<BF16>(cache + r * D * ES, at, D, v);
    }
  }
}

template <bool BF16, bool MX>
void launch_heads(const QkvArgs& a0, hipStream_t s) {
  QkvArgs a = a0;
  auto grid = [&](int hpw) {
    const int all = (a.n_q + hpw - 1) / hpw + 2 * ((a.n_kv + hpw - 1) / hpw);
    // wavefronts a row: the angles are formed once in each, but short runs of
    // steps start sooner (us a call, 1 / 2 / 4 / 5 wavefronts: 8192 rows 43 / 41 /
    // 49 / 53; 1 / 2 / 4 / 8 / 10: 1024 rows 12.4 / 9.6 / 9.5 / 9.6 / 11.8)
    const int parts = std::min(all, std::max(2, 4096 / std::max(a.T, 1)));
    a.steps = (all + parts - 1) / parts;
    return dim3(a.T, (all + a.steps - 1) / a.steps);
  };
  if (a.D <= 32) { const dim3 g = grid(16); qkv_cache_kernel<BF16, MX, 4><<<g, 64, 0, s>>>(a); }
  else if (a.D <= 64) { const dim3 g = grid(8); qkv_cache_kernel<BF16, MX, 8><<<g, 64, 0, s>>>(a); }
  else if (a.D <= 128) { const dim3 g = grid(4); qkv_cache_kernel<BF16, MX, 16><<<g, 64, 0, s>>>(a); }
  else { const dim3 g = grid(2); qkv_cache_kernel<BF16, MX, 32><<<g, 64, 0, s>>>(a); }
}

}  // namespace

hipError_t launch_qkv_cache(const void* qkv, bool bf16, int T, int n_q, int n_kv, int D, const float* q_norm,
                            const float* k_norm, float eps, const int32_t* positions, const float* inv_freq, int rot,
                            const int32_t* slot_map, bool mx, int n_pages, int page_size, void* q_out, void* k_cache,
                            void* v_cache, uint8_t* k_scale, uint8_t* v_scale, hipStream_t s) {
  const QkvArgs a{qkv,     q_norm,  k_norm, positions, inv_freq, slot_map, q_out, k_cache,   v_cache,
                  k_scale, v_scale, T,      n_q,       n_kv,     D,        rot,   n_pages, page_size, 0, eps};
  if (mx) launch_heads<true, true>(a, s);
  else if (bf16) launch_heads<true, false>(a, s);
  else launch_heads<false, false>(a, s);
  return hipGetLastError();
}

}  // namespace decomoe
