// Attention of one new token of each sequence over its paged cache.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c q.k_j - m),  c = scale log2 e
//
// One pass over keys and values with the running maximum m and sum.  The G
// query heads that share a key/value head are the 16 columns of the matrix
// instructions, so a cache row is read once for all of them, straight into
// registers: S^T = K Q^T leaves a head in each lane's column, and its terms
// are already the second operand of O^T = V^T P^T (the order of the keys
// inside a product is free); V^T is V's rows with neighbouring 16-bit values
// exchanged between registers.  Nothing passes through LDS until the join.
//
// Work: a tile is 4 x 16 KT keys of one (sequence, key/value head, 16 query
// heads).  All tiles, in that order, are cut into equal runs, one for each
// workgroup, whatever the lengths are; the four wavefronts take a tile's
// quarters.  A run that covers a whole segment writes its output; the others
// leave their sums in the workspace for a second launch that joins them in
// order.
#include "block.hpp"

#include <algorithm>

namespace decomoe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMaxSeq = 4096;
constexpr int kWaves = 4;
// workgroups that share the tiles: four on each of 256 compute units
constexpr int kRuns = 1024;

struct AttnArgs {
  const void *q, *k, *v;
  const uint8_t *ks, *vs;
  const int32_t *table, *lens;
  void* out;
  float* part;      // [2 kRuns][16 heads: m, l][...] then [2 kRuns][heads][D]
  float* part_o;
  int32_t* tiles;   // [n_seq + 1] exclusive sums of the sequences' tiles
  int n_seq, n_q, n_kv, G, blocks, max_pages, page, n_pages;  // blocks: of 16 query heads a key/value head
  uint32_t page_mul;
  int page_shift;
  float c;
};

// key / page for key < 2^31
__device__ __forceinline__ uint32_t page_of(const AttnArgs& a, uint32_t key) {
  return static_cast<uint32_t>(((uint64_t)key * a.page_mul) >> a.page_shift);
}

// the run that holds unit u of `units` over `runs`, and a run's first unit
__device__ __forceinline__ int run_of(long long u, long long units, long long runs) {
  return static_cast<int>(((u + 1) * runs - 1) / units);
}
__device__ __forceinline__ long long run_begin(long long r, long long units, long long runs) {
  return r * units / runs;
}

// KIND: MOE_F32, MOE_BF16 or kMx; D head length.
template <int KIND, int D>
struct Shape {
  static constexpr int KT = KIND == 0 ? 1 : 2;          // 16-key groups a wavefront step
  static constexpr int KEYS = 16 * KT;                  // keys of a step
  static constexpr int TILE = kWaves * KEYS;            // keys of a tile
  static constexpr int VC = D > 128 ? 2 : 1;            // column parts of V
  static constexpr int VD = D / (16 * VC);              // V columns of a lane and part
  static constexpr int ES = KIND == 0 ? 4 : KIND == 1 ? 2 : 1;
};

template <int KIND, int D>
__global__ __launch_bounds__(64 * kWaves) void attn_kernel(const AttnArgs a) {
  using S = Shape<KIND, D>;
  constexpr int KT = S::KT, VC = S::VC, VD = S::VD, ES = S::ES, KEYS = S::KEYS, TILE = S::TILE;
  constexpr int KS = KIND == 0 ? D / 16 : D / 32;  // K steps: 16 bytes (f32, bf16) or 8 (mx) a lane
  constexpr int OT = D / 16;                       // output tiles of 16 columns
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, c = lane & 15, g = lane >> 4;

  // exclusive sums of the sequences' tiles (a sequence without keys has one)
  int32_t* sums = reinterpret_cast<int32_t*>(lds);  // [n_seq + 1]
  const int cap = a.max_pages * a.page;
  {
    __shared__ int32_t wave_sum[kWaves];
    const int per = (a.n_seq + 255) / 256, s0 = tid * per;
    int mine = 0;
    for (int s = s0; s < min(s0 + per, a.n_seq); ++s) mine += max(1, (clampi(a.lens[s], 0, cap) - 1) / TILE + 1);
    int up = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(up, o, 64);
      if (lane >= o) up += u;
    }
    if (lane == 63) wave_sum[wv] = up;
    __syncthreads();
    int at = up - mine;
    for (int w = 0; w < wv; ++w) at += wave_sum[w];
    for (int s = s0; s < min(s0 + per, a.n_seq); ++s) {
      sums[s] = at;
      at += max(1, (clampi(a.lens[s], 0, cap) - 1) / TILE + 1);
    }
    if (tid == 255) sums[a.n_seq] = at;
    __syncthreads();
  }
  if (blockIdx.x == 0)
    for (int s = tid; s <= a.n_seq; s += 256) a.tiles[s] = sums[s];
  const int hb_all = a.n_kv * a.blocks;
  const long long units = (long long)sums[a.n_seq] * hb_all;
  const long long runs = min((long long)gridDim.x, units);
  if (blockIdx.x >= runs) return;
  long long u = run_begin(blockIdx.x, units, runs);
  const long long u_end = run_begin(blockIdx.x + 1, units, runs);

  const int hl = min(16, a.G);               // heads of a block
  float* lds_m = lds + ((a.n_seq + 4) & ~3);  // [kWaves][16] m, then l
  float* lds_l = lds_m + kWaves * 16;
  float* lds_o = lds_l + kWaves * 16;         // [kWaves][hl][D]

  while (u < u_end) {
    int s;
    {
      int lo = 0, hi = a.n_seq - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((long long)sums[mid] * hb_all <= u) lo = mid; else hi = mid - 1;
      }
      s = lo;
    }
    const int nt = sums[s + 1] - sums[s];
    const int rem = static_cast<int>(u - (long long)sums[s] * hb_all);
    const int hb = rem / nt, tile0 = rem % nt;
    const int tile1 = static_cast<int>(min((long long)nt, tile0 + (u_end - u)));
    const int kv = hb / a.blocks, h0 = kv * a.G + (hb % a.blocks) * 16;
    const int heads = min(16, a.G - (hb % a.blocks) * 16);
    const int len = clampi(a.lens[s], 0, cap);
    const int32_t* table = a.table + (size_t)s * a.max_pages;

    // this lane's part of its head's query: the second operand of S^T
    const char* qr = static_cast<const char*>(a.q) + ((size_t)s * a.n_q + h0 + c) * D * (KIND == 0 ? 4 : 2);
    uint4 q[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i)
      q[i] = c < heads ? *reinterpret_cast<const uint4*>(qr + i * 64 + g * 16) : make_uint4(0, 0, 0, 0);

    float m = -INFINITY, l = 0.f;
    f32x4 o[OT];
#pragma unroll
    for (int i = 0; i < OT; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    // cache row of key `key` (page * n_kv + head) * page_size + slot, ~0 if there is none
    auto row_of = [&](int key) -> uint32_t {
      if (key >= len) return ~0u;
      const uint32_t p = page_of(a, key);
      const int pg = table[p];
      if (pg < 0 || pg >= a.n_pages) return ~0u;
      return ((uint32_t)pg * a.n_kv + kv) * a.page + ((uint32_t)key - p * a.page);
    };
    int key0 = tile0 * TILE + wv * KEYS;
    uint32_t next = tile0 < tile1 ? row_of(key0 + (lane & (KEYS - 1))) : ~0u;
    for (int tile = tile0; tile < tile1; ++tile, key0 += TILE) {
      const uint32_t row = next;
      const uint32_t there = static_cast<uint32_t>(__ballot(row != ~0u));  // bit j: key j of the step (lanes repeat)
      if (tile + 1 < tile1) next = row_of(key0 + TILE + (lane & (KEYS - 1)));
      if ((there & ((KEYS == 32) ? ~0u : (1u << (KEYS & 31)) - 1u)) == 0) continue;
      const uint32_t safe = row == ~0u ? 0u : row;

      // S^T = K Q^T
      f32x4 sc[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const size_t r = static_cast<uint32_t>(__shfl(static_cast<int>(safe), t * 16 + c, 64));
        const char* kr = static_cast<const char*>(a.k) + r * (D * ES);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          if constexpr (KIND == 1) {
            const uint4 kk = *reinterpret_cast<const uint4*>(kr + i * 64 + g * 16);
            sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk),
                                                            __builtin_bit_cast(bf16x8, q[i]), sc[t], 0, 0, 0);
          } else if constexpr (KIND == 0) {
            const float4 kk = *reinterpret_cast<const float4*>(kr + i * 64 + g * 16);
            const float ka[4] = {kk.x, kk.y, kk.z, kk.w};
            const uint32_t qa[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[e], __uint_as_float(qa[e]), sc[t], 0, 0, 0);
          } else {
            const uint2 kk = *reinterpret_cast<const uint2*>(kr + i * 32 + g * 8);
            const uint32_t b = a.ks[r * (D / 32) + i];
            const float f = b == 255u ? __uint_as_float(0x7fc00000u) : mx_scale(b);
            const bf16x2_t k0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kk.x, f, false);
            const bf16x2_t k1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kk.x, f, true);
            const bf16x2_t k2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kk.y, f, false);
            const bf16x2_t k3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kk.y, f, true);
            const bf16x8 ka = {k0[0], k0[1], k1[0], k1[1], k2[0], k2[1], k3[0], k3[1]};
            sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, __builtin_bit_cast(bf16x8, q[i]), sc[t], 0, 0, 0);
          }
        }
      }

      // running maximum and sum; lane: head c, keys 16 t + 4 g + i
      float top = m;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[t][i] = (there >> (t * 16 + g * 4 + i)) & 1u ? sc[t][i] * a.c : -INFINITY;
          top = fmaxf(top, sc[t][i]);
        }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float ref = top == -INFINITY ? 0.f : top;  // nothing yet: every term is 0
      const float keep = __builtin_amdgcn_exp2f(m - ref);
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float p = __builtin_amdgcn_exp2f(sc[t][i] - ref);
          if constexpr (KIND != 0) p = bf16_to_f32(f32_to_bf16(p));  // the weight that v gets
          sc[t][i] = p;
          sum += p;
        }
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      l = l * keep + sum;
      m = top;
#pragma unroll
      for (int i = 0; i < OT; ++i) o[i] *= keep;

      // O^T += V^T P^T: the keys of a product in the order 16 t + 4 g + i
      uint32_t vr[KT * 4];
#pragma unroll
      for (int j = 0; j < KT * 4; ++j)
        vr[j] = static_cast<uint32_t>(__shfl(static_cast<int>(safe), (j >> 2) * 16 + g * 4 + (j & 3), 64));
      const bool whole = there == ~0u || (KEYS < 32 && (there & ((1u << (KEYS & 31)) - 1u)) == (1u << (KEYS & 31)) - 1u);
#pragma unroll
      for (int part = 0; part < VC; ++part) {
        const int col = part * (D / 2) + c * VD;  // this lane's first column of the part
        if constexpr (KIND == 0) {
          float vv[4][VD];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const char* p = static_cast<const char*>(a.v) + (size_t)vr[j] * (D * ES) + col * ES;
            struct alignas(4) Row { float f[VD]; };
            const Row rw = load_raw<Row>(p);
            const bool ok = whole || ((there >> (g * 4 + j)) & 1u);
#pragma unroll
            for (int e = 0; e < VD; ++e) vv[j][e] = ok ? rw.f[e] : 0.f;
          }
#pragma unroll
          for (int e = 0; e < VD; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[part * VD + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[j][e], sc[0][j], o[part * VD + e], 0, 0, 0);
        } else {
          const bf16x8 pb = __builtin_bit_cast(
              bf16x8, make_uint4(pack_bf16x2(sc[0][0], sc[0][1]), pack_bf16x2(sc[0][2], sc[0][3]),
                                 pack_bf16x2(sc[KT - 1][0], sc[KT - 1][1]), pack_bf16x2(sc[KT - 1][2], sc[KT - 1][3])));
          uint32_t vv[8][VD / 2];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool ok = whole || ((there >> ((j >> 2) * 16 + g * 4 + (j & 3))) & 1u);
            const char* p = static_cast<const char*>(a.v) + (size_t)vr[j] * (D * ES) + col * ES;
            if constexpr (KIND == 1) {
              struct alignas(4) Row { uint32_t w[VD / 2]; };
              const Row rw = load_raw<Row>(p);
#pragma unroll
              for (int e = 0; e < VD / 2; ++e) vv[j][e] = ok ? rw.w[e] : 0u;
            } else {
              struct alignas(2) Row { uint16_t w[VD / 2]; };
              const Row rw = load_raw<Row>(p);
              // a lane's columns may span two blocks of 32 (VD = 6)
#pragma unroll
              for (int e = 0; e < VD / 2; ++e) {
                const uint32_t b = a.vs[(size_t)vr[j] * (D / 32) + (col + 2 * e) / 32];
                const float f = b == 255u ? __uint_as_float(0x7fc00000u) : mx_scale(b);
                const bf16x2_t w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(rw.w[e], f, false);
                vv[j][e] = ok ? __builtin_bit_cast(uint32_t, w) : 0u;
              }
            }
          }
#pragma unroll
          for (int e = 0; e < VD / 2; ++e) {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              lo[j] = __builtin_amdgcn_perm(vv[2 * j + 1][e], vv[2 * j][e], 0x05040100u);
              hi[j] = __builtin_amdgcn_perm(vv[2 * j + 1][e], vv[2 * j][e], 0x07060302u);
            }
            const int x = part * VD + 2 * e;
            o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), pb, o[x], 0, 0, 0);
            o[x + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), pb, o[x + 1], 0, 0, 0);
          }
        }
      }
    }

    // join the four wavefronts.  Lane: head c; o[part * VD + e][i] is column
    // part * D / 2 + (4 g + i) * VD + e
    if (g == 0) {
      lds_m[wv * 16 + c] = m;
      lds_l[wv * 16 + c] = l;
    }
    __syncthreads();
    float top = lds_m[c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds_m[w * 16 + c]);
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    if (c < heads)
#pragma unroll
      for (int x = 0; x < OT; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          lds_o[(wv * hl + c) * D + (x / VD) * (D / 2) + (4 * g + i) * VD + x % VD] = o[x][i] * f;
    __syncthreads();
    const bool first = tile0 == 0, end = tile1 == nt;
    const size_t slot = 2 * (size_t)blockIdx.x + (first ? 1 : 0);  // of a partial result
    for (int i = tid; i < heads * D; i += 256) {
      const int h = i / D;
      float top = lds_m[h];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds_m[w * 16 + h]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, v = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        sum += lds_l[w * 16 + h] * __builtin_amdgcn_exp2f(lds_m[w * 16 + h] - ref);
        v += lds_o[w * hl * D + i];
      }
      if (first && end) {
        const float r = sum == 0.f ? 0.f : v / sum;
        const size_t at = ((size_t)s * a.n_q + h0) * D + i;
        if constexpr (KIND == 0) static_cast<float*>(a.out)[at] = r;
        else static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(r);
      } else {
        a.part_o[slot * 16 * D + i] = v;
        if (i % D == 0) {
          a.part[slot * 32 + h] = top;
          a.part[slot * 32 + 16 + h] = sum;
        }
      }
    }
    __syncthreads();
    u += tile1 - tile0;
  }
}

// the partial results of segments that several runs share, in order; a
// workgroup a (segment, head)
template <bool BF16>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs a, int D, int runs_max) {
  __shared__ float acc[4][256];
  const int hb_all = a.n_kv * a.blocks;
  const int seg = blockIdx.x, h = blockIdx.y, s = seg / hb_all, hb = seg % hb_all;
  const int heads = min(16, a.G - (hb % a.blocks) * 16);
  if (h >= heads) return;
  const int nt = a.tiles[s + 1] - a.tiles[s];
  const long long units = (long long)a.tiles[a.n_seq] * hb_all, runs = min((long long)runs_max, units);
  const long long u0 = (long long)a.tiles[s] * hb_all + (long long)hb * nt;
  const int r0 = run_of(u0, units, runs), r1 = run_of(u0 + nt - 1, units, runs);
  if (r0 == r1) return;  // one run wrote the output
  auto slot = [&](int r) -> size_t { return 2 * (size_t)r + (r == r0 ? 1 : 0); };
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  float top = -INFINITY;
  for (int r = r0 + lane; r <= r1; r += 64) top = fmaxf(top, a.part[slot(r) * 32 + h]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int r = r0; r <= r1; ++r) sum += a.part[slot(r) * 32 + 16 + h] * __builtin_amdgcn_exp2f(a.part[slot(r) * 32 + h] - ref);
  for (int d0 = 0; d0 < D; d0 += 64) {
    const int d = d0 + lane;
    float v = 0.f;
    if (d < D)
      for (int r = r0 + wv; r <= r1; r += 4)
        v += a.part_o[(slot(r) * 16 + h) * D + d] * __builtin_amdgcn_exp2f(a.part[slot(r) * 32 + h] - ref);
    acc[wv][d0 / 64 * 64 + lane] = v;
  }
  __syncthreads();
  if (tid < D) {
    const float v = (acc[0][tid] + acc[1][tid]) + (acc[2][tid] + acc[3][tid]);
    const float r = sum == 0.f ? 0.f : v / sum;
    const size_t at = ((size_t)s * a.n_q + (hb / a.blocks) * a.G + (hb % a.blocks) * 16 + h) * D + tid;
    if constexpr (BF16) static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(r);
    else static_cast<float*>(a.out)[at] = r;
  }
}

template <int KIND, int D>
hipError_t launch_d(const AttnArgs& a, int max_keys, hipStream_t s) {
  using S = Shape<KIND, D>;
  const long long tiles = std::max(1, (max_keys - 1) / S::TILE + 1);
  const long long most = tiles * a.n_seq * a.n_kv * a.blocks;
  const int grid = (int)std::min<long long>(kRuns, most);
  const size_t lds = ((size_t)((a.n_seq + 4) & ~3) + 2 * kWaves * 16 + (size_t)kWaves * std::min(a.G, 16) * D) * 4;
  attn_kernel<KIND, D><<<grid, 64 * kWaves, lds, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || tiles == 1) return e;  // (a segment of one tile is never cut)
  attn_join_kernel<KIND != 0><<<dim3(a.n_seq * a.n_kv * a.blocks, std::min(a.G, 16)), 256, 0, s>>>(a, D, grid);
  return hipGetLastError();
}

template <int KIND>
hipError_t launch_kind(const AttnArgs& a, int D, int max_keys, hipStream_t s) {
  switch (D) {
    case 32: return launch_d<KIND, 32>(a, max_keys, s);
    case 64: return launch_d<KIND, 64>(a, max_keys, s);
    case 96: return launch_d<KIND, 96>(a, max_keys, s);
    case 128: return launch_d<KIND, 128>(a, max_keys, s);
    case 192: return launch_d<KIND, 192>(a, max_keys, s);
    default: return launch_d<KIND, 256>(a, max_keys, s);
  }
}

size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace

bool attn_sizes_ok(int n_seq, int n_q, int n_kv, int D, int max_keys) {
  if (D != 32 && D != 64 && D != 96 && D != 128 && D != 192 && D != 256) return false;
  if (n_seq > kMaxSeq) return false;
  const long long blocks = (n_q / n_kv + 15) / 16;
  const long long segments = (long long)n_seq * n_kv * blocks;
  return segments <= INT32_MAX && (long long)((max_keys - 1) / 64 + 1) <= INT32_MAX / std::max(1LL, segments);
}

size_t attn_ws_bytes(int n_seq, int n_q, int n_kv, int D, int max_keys) {
  (void)max_keys;
  (void)n_q;
  (void)n_kv;
  return up256((size_t)(n_seq + 1) * 4) + up256((size_t)2 * kRuns * 32 * 4) + (size_t)2 * kRuns * 16 * D * 4;
}

hipError_t launch_attn_decode(const void* q, int kind, int n_seq, int n_q, int n_kv, int D, const void* k_cache,
                              const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int n_pages,
                              int page_size, const int32_t* block_table, int max_pages, const int32_t* lens,
                              float scale, void* out, void* ws, hipStream_t s) {
  char* w = static_cast<char*>(ws);
  AttnArgs a{};
  a.q = q, a.k = k_cache, a.v = v_cache, a.ks = k_scale, a.vs = v_scale;
  a.table = block_table, a.lens = lens, a.out = out;
  a.tiles = reinterpret_cast<int32_t*>(w);
  a.part = reinterpret_cast<float*>(w + up256((size_t)(n_seq + 1) * 4));
  a.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(a.part) + up256((size_t)2 * kRuns * 32 * 4));
  a.n_seq = n_seq, a.n_q = n_q, a.n_kv = n_kv, a.G = n_q / n_kv, a.blocks = (a.G + 15) / 16;
  a.max_pages = max_pages, a.page = page_size, a.n_pages = n_pages;
  // exact division of a 31-bit key: mul = ceil(2^(31 + b) / page), 2^b >= page
  int b = 0;
  while ((1LL << b) < page_size) ++b;
  a.page_shift = 31 + b;
  a.page_mul = static_cast<uint32_t>(((1ULL << (31 + b)) + page_size - 1) / page_size);
  a.c = scale * 1.4426950408889634f;
  const int max_keys = max_pages * page_size;
  if (kind == 0) return launch_kind<0>(a, D, max_keys, s);
  if (kind == 1) return launch_kind<1>(a, D, max_keys, s);
  return launch_kind<kMx>(a, D, max_keys, s);
}

}  // namespace decomoe
