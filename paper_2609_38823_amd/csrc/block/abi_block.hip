// Exported C ABI of the attention half of a block: host-side validation, then
// the launches.  Nothing here allocates, frees or synchronises.
#include <math.h>

#include "block.hpp"

#include "../../../include/decomoe_block.h"
#include "../checks.hpp"

namespace {

using namespace decomoe::checks;

static_assert(BLK_MX8 == decomoe::kMx && MOE_BF16 == 1 && MOE_F32 == 0, "kinds of the header and the kernels agree");

constexpr int kMaxD = 32768;       // blk_rms_norm's longest row
constexpr int kMaxCount = 1 << 30;  // rows and table entries that kernels count with a step in 32 bits
constexpr int kMaxWaves = 1 << 25;  // a launch counts its threads in 32 bits
constexpr int kMaxRows = 1 << 22;   // blk_linear_w4's rows (64 a workgroup row of at most 65536)
constexpr int kMaxK = 1 << 24;      // and columns (64 rows are addressed with 32 bits)
constexpr int kMaxN = 1 << 26;      // and weight rows (512 threads for 16)

Range none() { return Range{0, 0}; }
Range opt(const void* p, size_t bytes) { return p ? rng(p, bytes) : none(); }
bool same(const void* a, const void* b) { return a && a == b; }
bool above(long long a, long long b, long long limit) { return a > limit / (b > 0 ? b : 1); }
bool good_eps(double eps) { return eps >= 0.0 && isfinite(static_cast<float>(eps)); }

// the paged cache: what both of its functions ask of its sizes
int cache_status(moe_dtype dtype, int cache_dtype, int n_kv, int D, int n_pages, int page_size,
                 const uint8_t* k_scale, const uint8_t* v_scale) {
  if (!valid_dtype(dtype) || n_kv < 1 || D < 1 || n_pages < 1 || page_size < 1) return MOE_EINVAL;
  if (cache_dtype != (int)dtype && cache_dtype != BLK_MX8) return MOE_EINVAL;
  if (cache_dtype == BLK_MX8 && dtype != MOE_BF16) return MOE_EUNSUPPORTED;
  if ((cache_dtype == BLK_MX8) != (k_scale != nullptr) || (cache_dtype == BLK_MX8) != (v_scale != nullptr))
    return MOE_EINVAL;
  if (above(n_pages, page_size, INT32_MAX)) return MOE_EUNSUPPORTED;
  return MOE_OK;
}
size_t cache_bytes(int cache_dtype, int n_kv, int D, int n_pages, int page_size) {
  return (size_t)n_pages * page_size * n_kv * D * (cache_dtype == BLK_MX8 ? 1 : elt_size((moe_dtype)cache_dtype));
}
size_t scale_bytes(int n_kv, int D, int n_pages, int page_size) {
  return (size_t)n_pages * page_size * n_kv * (D / 32);
}

}  // namespace

extern "C" {

int blk_rms_norm(const void* x, moe_dtype dtype, const void* residual, const float* weight, int T, int d, double eps,
                 void* h_out, void* y, void* q, uint8_t* q_scale, hipStream_t stream) {
  if (!valid_dtype(dtype) || T < 0 || d < 1 || !good_eps(eps)) return MOE_EINVAL;
  if (d > kMaxD || T > kMaxWaves / (d <= 512 ? 1 : d <= 4096 ? 4 : 16)) return MOE_EUNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!x || (q != nullptr) != (q_scale != nullptr) || (!h_out && !y && !q)) return MOE_EINVAL;
  if (!aligned_all({x, residual, weight, h_out, y, q, q_scale})) return MOE_EINVAL;
  const size_t row = (size_t)T * d * elt_size(dtype);
  Range o_h = opt(h_out, row), o_y = opt(y, row), o_q = opt(q, (size_t)T * d);
  Range o_s = opt(q_scale, (size_t)T * ((d + 31) / 32));
  Range in_x = rng(x, row), in_r = opt(residual, row), in_w = opt(weight, (size_t)d * 4);
  // a row is read whole before any of it is written: h_out or y in place
  auto placed = [&](void* o, Range r) {
    return (!overlap(r, in_x) || same(o, x)) && (!overlap(r, in_r) || same(o, residual));
  };
  if (any_alias({o_h, o_y, o_q, o_s}, {in_w}) || any_alias({o_q, o_s}, {in_x, in_r}) || !placed(h_out, o_h) ||
      !placed(y, o_y))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_rms_norm(x, dtype == MOE_BF16, residual, weight, T, d, static_cast<float>(eps),
                                             h_out, y, q, q_scale, stream));
}

int blk_kv_extend(const int32_t* len_in, const int32_t* add, int n_seq, int page_size, int max_pages, int n_pages,
                  int rows_max, const int32_t* n_free_in, int32_t* block_table, int32_t* free_pages,
                  int32_t* len_out, int32_t* n_free_out, int32_t* row_offsets, int32_t* slot_map,
                  int32_t* positions, int32_t* accepted, int32_t* status, hipStream_t stream) {
  if (n_seq < 0 || page_size < 1 || max_pages < 1 || n_pages < 1 || rows_max < 0) return MOE_EINVAL;
  if (above(n_pages, page_size, INT32_MAX) || above(max_pages, page_size, INT32_MAX) ||
      above(n_seq, max_pages, kMaxCount) || rows_max > kMaxCount)
    return MOE_EUNSUPPORTED;
  if (!n_free_in || !free_pages || !n_free_out || !row_offsets || !status) return MOE_EINVAL;
  if (n_seq > 0 && (!len_in || !add || !block_table || !len_out || !accepted)) return MOE_EINVAL;
  if (rows_max > 0 && (!slot_map || !positions)) return MOE_EINVAL;
  if (!aligned_all({len_in, add, n_free_in, block_table, free_pages, len_out, n_free_out, row_offsets, slot_map,
                    positions, accepted, status}))
    return MOE_EINVAL;
  const size_t n4 = (size_t)n_seq * 4, r4 = (size_t)rows_max * 4;
  Range o_l = rng(len_out, n4), o_f = rng(n_free_out, 4), in_l = rng(len_in, n4), in_f = rng(n_free_in, 4);
  if (same(len_out, len_in)) in_l = none();
  if (same(n_free_out, n_free_in)) in_f = none();
  if (any_alias({o_l, o_f, rng(block_table, n4 * max_pages), rng(free_pages, (size_t)n_pages * 4),
                 rng(row_offsets, n4 + 4), rng(slot_map, r4), rng(positions, r4), rng(accepted, n4),
                 rng(status, 16)},
                {in_l, in_f, rng(add, n4)}))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_kv_extend(len_in, add, n_seq, page_size, max_pages, n_pages, rows_max, n_free_in,
                                              block_table, free_pages, len_out, n_free_out, row_offsets, slot_map,
                                              positions, accepted, status, stream));
}

int blk_qkv_cache(const void* qkv, moe_dtype dtype, int T, int n_q, int n_kv, int D, const float* q_norm,
                  const float* k_norm, double eps, const int32_t* positions, const float* inv_freq, int rot,
                  const int32_t* slot_map, int cache_dtype, int n_pages, int page_size, void* q_out, void* k_cache,
                  void* v_cache, uint8_t* k_scale, uint8_t* v_scale, hipStream_t stream) {
  if (T < 0 || n_q < 1 || rot < 0 || rot > D || !good_eps(eps)) return MOE_EINVAL;
  int st = cache_status(dtype, cache_dtype, n_kv, D, n_pages, page_size, k_scale, v_scale);
  if (st != MOE_OK) return st;
  if (D % 32 != 0 || D > 256 || rot % 16 != 0 || n_q > 16384 || n_kv > 16384 || T > kMaxWaves)
    return MOE_EUNSUPPORTED;
  if (rot > 0 && T > 0 && (!positions || !inv_freq)) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!qkv || !slot_map || !q_out || !k_cache || !v_cache) return MOE_EINVAL;
  if (!aligned_all({qkv, q_norm, k_norm, positions, inv_freq, slot_map, q_out, k_cache, v_cache, k_scale, v_scale}))
    return MOE_EINVAL;
  const int es = elt_size(dtype);
  const size_t cb = cache_bytes(cache_dtype, n_kv, D, n_pages, page_size);
  const size_t sb = scale_bytes(n_kv, D, n_pages, page_size);
  if (any_alias({rng(q_out, (size_t)T * n_q * D * es), rng(k_cache, cb), rng(v_cache, cb), opt(k_scale, sb),
                 opt(v_scale, sb)},
                {rng(qkv, (size_t)T * (n_q + 2 * n_kv) * D * es), opt(q_norm, (size_t)D * 4),
                 opt(k_norm, (size_t)D * 4), rot ? rng(positions, (size_t)T * 4) : none(),
                 rot ? rng(inv_freq, (size_t)rot * 2) : none(), rng(slot_map, (size_t)T * 4)}))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_qkv_cache(qkv, dtype == MOE_BF16, T, n_q, n_kv, D, q_norm, k_norm,
                                              static_cast<float>(eps), positions, inv_freq, rot, slot_map,
                                              cache_dtype == BLK_MX8, n_pages, page_size, q_out, k_cache, v_cache,
                                              k_scale, v_scale, stream));
}

size_t blk_attn_workspace_size(int n_seq, int n_q, int n_kv, int D, int max_keys) {
  if (n_seq < 0 || n_q < 1 || n_kv < 1 || n_q % n_kv != 0 || D < 1 || max_keys < 1) return 0;
  if (!decomoe::attn_sizes_ok(n_seq, n_q, n_kv, D, max_keys)) return 0;
  return decomoe::attn_ws_bytes(n_seq, n_q, n_kv, D, max_keys);
}

int blk_attn_decode(const void* q, moe_dtype dtype, int n_seq, int n_q, int n_kv, int D, const void* k_cache,
                    const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int cache_dtype,
                    int n_pages, int page_size, const int32_t* block_table, int max_pages, const int32_t* lens,
                    double scale, void* out, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (n_seq < 0 || n_q < 1 || max_pages < 1 || !isfinite(static_cast<float>(scale * 1.4426950408889634)))
    return MOE_EINVAL;
  int st = cache_status(dtype, cache_dtype, n_kv, D, n_pages, page_size, k_scale, v_scale);
  if (st != MOE_OK) return st;
  if (n_q % n_kv != 0) return MOE_EINVAL;
  if (above(max_pages, page_size, INT32_MAX) ||
      !decomoe::attn_sizes_ok(n_seq, n_q, n_kv, D, max_pages * page_size) ||
      (unsigned long long)n_pages * page_size > (UINT32_MAX - 1ull) / n_kv)
    return MOE_EUNSUPPORTED;
  if (n_seq == 0) return MOE_OK;
  if (!q || !k_cache || !v_cache || !block_table || !lens || !out) return MOE_EINVAL;
  if (!aligned_all({q, k_cache, v_cache, k_scale, v_scale, block_table, lens, out, ws})) return MOE_EINVAL;
  const size_t need = decomoe::attn_ws_bytes(n_seq, n_q, n_kv, D, max_pages * page_size);
  if (!ws || ws_bytes < need) return MOE_EWORKSPACE;
  const size_t qb = (size_t)n_seq * n_q * D * elt_size(dtype);
  const size_t cb = cache_bytes(cache_dtype, n_kv, D, n_pages, page_size);
  const size_t sb = scale_bytes(n_kv, D, n_pages, page_size);
  if (any_alias({rng(out, qb), rng(ws, need)},
                {rng(q, qb), rng(k_cache, cb), rng(v_cache, cb), opt(k_scale, sb), opt(v_scale, sb),
                 rng(block_table, (size_t)n_seq * max_pages * 4), rng(lens, (size_t)n_seq * 4)}))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_attn_decode(q, cache_dtype, n_seq, n_q, n_kv, D, k_cache, v_cache, k_scale,
                                                v_scale, n_pages, page_size, block_table, max_pages, lens,
                                                static_cast<float>(scale), out, ws, stream));
}

int blk_linear_w4(const void* x, int x_dtype, const uint8_t* x_scale, int T, int k, const uint8_t* codes,
                  const uint8_t* scales, int n, void* y, moe_dtype y_dtype, hipStream_t stream) {
  if ((x_dtype != MOE_F32 && x_dtype != MOE_BF16 && x_dtype != BLK_MX8) || !valid_dtype(y_dtype)) return MOE_EINVAL;
  if (T < 0 || n < 1 || k < 1) return MOE_EINVAL;
  if (k % 32 != 0 || T > kMaxRows || k > kMaxK || n > kMaxN) return MOE_EUNSUPPORTED;
  if (!codes || !scales) return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!x || !y || (x_dtype == BLK_MX8) != (x_scale != nullptr)) return MOE_EINVAL;
  if (!aligned_all({x, x_scale, codes, scales, y})) return MOE_EINVAL;
  const int xs = x_dtype == BLK_MX8 ? 1 : elt_size((moe_dtype)x_dtype);
  if (any_alias({rng(y, (size_t)T * n * elt_size(y_dtype))},
                {rng(x, (size_t)T * k * xs), opt(x_scale, (size_t)T * (k / 32)), rng(codes, (size_t)n * (k / 2)),
                 rng(scales, (size_t)n * (k / 32))}))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_linear_w4(x, x_dtype, x_scale, T, k, codes, scales, n, y, y_dtype == MOE_BF16,
                                              stream));
}

int blk_quantize_w4(const void* w, moe_dtype dtype, int n, int k, uint8_t* codes, uint8_t* scales,
                    hipStream_t stream) {
  if (!valid_dtype(dtype) || n < 1 || k < 1) return MOE_EINVAL;
  if (k % 32 != 0) return MOE_EUNSUPPORTED;
  if (!w || !codes || !scales) return MOE_EINVAL;
  if (!aligned_all({w, codes, scales})) return MOE_EINVAL;
  if (any_alias({rng(codes, (size_t)n * (k / 2)), rng(scales, (size_t)n * (k / 32))},
                {rng(w, (size_t)n * k * elt_size(dtype))}))
    return MOE_EALIAS;
  return hip_status(decomoe::launch_quantize_w4(w, dtype == MOE_BF16, n, k, codes, scales, stream));
}

}  // extern "C"
