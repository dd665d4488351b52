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
#include "block.hpp"

namespace decomoe {
namespace {

struct QkvArgs {
  const void* qkv;
  const float *q_norm, *k_norm;
  const int32_t* positions;
  const float* inv_freq;
  const int32_t* slot_map;
  void *q_out, *k_cache, *v_cache;
  uint8_t *k_scale, *v_scale;
  int T, n_q, n_kv, D, rot, n_pages, page, heads;  // heads: of one wavefront's share (a multiple of its groups)
  float eps;
};

template <bool BF16, bool MX, int GL>
__global__ __launch_bounds__(64) void qkv_cache_kernel(const QkvArgs a) {
  constexpr int HPW = 64 / GL, ES = BF16 ? 2 : 4;
  const int lane = threadIdx.x, l = lane % GL, D = a.D, at = l * 8;
  const int t = blockIdx.x, n_all = a.n_q + 2 * a.n_kv, half = a.rot / 2;
  const bool on = at < D;  // lanes beyond the head's length
  const int slot = a.slot_map[t];
  const bool kept = slot >= 0 && slot / a.page < a.n_pages;
  const int pg = kept ? slot / a.page : 0, off = kept ? slot % a.page : 0;

  // this lane's rotation: partner column, cosines, signed sines
  const bool turned = at < a.rot;
  const int pair = at < half ? at + half : at - half;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) cs[e] = 1.f, sn[e] = 0.f;
  if (turned) {
    const double p = static_cast<double>(a.positions[t]);
    const int j = at < half ? at : at - half;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      double u = p * static_cast<double>(a.inv_freq[j + e]) * 0.15915494309189533577;  // in turns
      u -= rint(u);
      sincospif(2.f * static_cast<float>(u), &sn[e], &cs[e]);
      if (at < half) sn[e] = -sn[e];
    }
  }
  float w[2][8] = {}, wp[2][8] = {};
  auto weights = [&](const float* n, float (&wv)[8], float (&wpv)[8]) {
    if (!n || !on) return;
    load8<false>(n, at, D, wv);
    if (turned) load8<false>(n, pair, D, wpv);
  };
  weights(a.q_norm, w[0], wp[0]);
  weights(a.k_norm, w[1], wp[1]);

  const int h_end = min(n_all, ((int)blockIdx.y + 1) * a.heads);
  for (int h = blockIdx.y * a.heads + lane / GL; h < h_end; h += HPW) {
    const char* src = static_cast<const char*>(a.qkv) + ((size_t)t * n_all + h) * D * ES;
    const int kind = h < a.n_q ? 0 : h < a.n_q + a.n_kv ? 1 : 2;
    float v[8] = {}, u[8] = {};
    if (on) load8<BF16>(src, at, D, v);
    if (kind < 2) {
      if (on && turned) load8<BF16>(src, pair, D, u);
      if (kind ? a.k_norm != nullptr : a.q_norm != nullptr) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
#pragma unroll
        for (int o = GL / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
        const float f = 1.f / sqrtf(sum / static_cast<float>(D) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = v[e] * f * (kind ? w[1][e] : w[0][e]);
          u[e] = u[e] * f * (kind ? wp[1][e] : wp[0][e]);
        }
      }
      if (turned)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], cs[e], u[e] * sn[e]);
    }
    if (kind == 0) {
      if (on) store8<BF16>(static_cast<char*>(a.q_out) + ((size_t)t * a.n_q + h) * D * ES, at, D, v);
      continue;
    }
    const int hk = h - a.n_q - (kind == 2 ? a.n_kv : 0);
    const size_t r = ((size_t)pg * a.n_kv + hk) * a.page + off;
    char* cache = static_cast<char*>(kind == 1 ? a.k_cache : a.v_cache);
    if constexpr (MX) {
      const uint32_t byte = mx8_byte(block_most(v));
      if (kept && on) {
        store_raw(cache + r * D + at, to_e4m3x8(v, mx_inverse(byte)));
        if ((l & 3) == 0) (kind == 1 ? a.k_scale : a.v_scale)[r * (D / 32) + l / 4] = static_cast<uint8_t>(byte);
      }
    } else {
      if (kept && on) store8<BF16>(cache + r * D * ES, at, D, v);
    }
  }
}

template <bool BF16, bool MX>
void launch_heads(const QkvArgs& a0, hipStream_t s) {
  QkvArgs a = a0;
  const int n_all = a.n_q + 2 * a.n_kv;
  // heads a wavefront: all of a row's where the rows alone fill the card
  // (the angles are formed once), one step of each group where they do not
  auto share = [&](int hpw) {
    const int parts = a.T >= 4096 ? 1 : n_all;
    a.heads = (n_all + parts * hpw - 1) / (parts * hpw) * hpw;
    return dim3(a.T, (n_all + a.heads - 1) / a.heads);
  };
  if (a.D <= 32) { const dim3 g = share(16); qkv_cache_kernel<BF16, MX, 4><<<g, 64, 0, s>>>(a); }
  else if (a.D <= 64) { const dim3 g = share(8); qkv_cache_kernel<BF16, MX, 8><<<g, 64, 0, s>>>(a); }
  else if (a.D <= 128) { const dim3 g = share(4); qkv_cache_kernel<BF16, MX, 16><<<g, 64, 0, s>>>(a); }
  else { const dim3 g = share(2); qkv_cache_kernel<BF16, MX, 32><<<g, 64, 0, s>>>(a); }
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
