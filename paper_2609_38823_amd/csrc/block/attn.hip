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
// order.  Where a segment is a few tiles, a workgroup takes it whole.
//
// Bound: memory, with the next step's rows always in flight.  64 sequences of
// 1 to 8192 keys, 4 heads of 128, bf16: 104 us with the join for 0.54 GB (5.2
// TB/s); one sequence of 131072 keys: bf16 52 us (268 MB, 5.2 TB/s), 8-bit 33
// us (138 MB; the conversions and the start and end of a run show).
#include "block.hpp"

#include <algorithm>

namespace decomoe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMaxSeq = 4096;
constexpr int W = 4;  // wavefronts a workgroup
// workgroups that share the tiles, at most: four on each of 256 compute units
constexpr int kRuns = 1024;

struct AttnArgs {
  const void *q, *k, *v;
  const uint8_t *ks, *vs;
  const int32_t *table, *lens;
  void* out;
  float* part;      // [2 kRuns][16 heads: m, l][...] then [2 kRuns][heads][D]
  float* part_o;
  int32_t* shared;  // [segments][2] the first and the last run of a segment
  int n_seq, n_q, n_kv, G, blocks, max_pages, page, n_pages;  // blocks: of 16 query heads a key/value head
  uint32_t page_mul;
  int page_shift;
  float c;
};

// key / page for key < 2^31
__device__ __forceinline__ uint32_t page_of(const AttnArgs& a, uint32_t key) {
  return static_cast<uint32_t>(((uint64_t)key * a.page_mul) >> a.page_shift);
}

// the first unit of run r: `units` in `runs` parts, the first of them one longer
__device__ __forceinline__ uint32_t run_begin(uint32_t r, uint32_t units, uint32_t runs) {
  return r * (units / runs) + min(r, units % runs);
}

// KIND: MOE_F32, MOE_BF16 or kMx; D head length.
template <int KIND, int D>
struct Shape {
  static constexpr int KT = KIND == 0 ? 1 : 2;          // 16-key groups of a wavefront's step
  static constexpr int KEYS = 16 * KT;                  // keys of a step
  static constexpr int TILE = W * KEYS;                 // keys of a tile
  static constexpr int VC = D > 128 ? 2 : 1;            // column parts of V
  static constexpr int VD = D / (16 * VC);              // V columns of a lane and part
  static constexpr int ES = KIND == 0 ? 4 : KIND == 1 ? 2 : 1;
  static constexpr int KS = KIND == 0 ? D / 16 : D / 32;  // products of S^T: 16 or 32 columns each
  static constexpr bool WIDE = KIND == kMx && D % 64 == 0;  // 16-byte loads of 8-bit keys: two products a load
  // a lane's loads of a key's row, and how far apart they are
  static constexpr int KL = WIDE ? KS / 2 : KS, KB = KIND == kMx && !WIDE ? 8 : 16, KSTEP = 4 * KB;
  static constexpr int VW = (VD * ES + 3) / 4;          // words of a lane's part of a value row
  static constexpr int NS = D / 32, NW = (NS + 3) / 4;  // scales of a row (kMx), and their words
  // workgroups that a compute unit's registers hold
  static constexpr int PER_CU = D >= 192 ? 1 : D == 128 ? 2 : D == 96 ? (KIND == 0 ? 3 : 2) : D == 64 ? 3 : 4;
};

// what a lane loads for one step of 16 KT keys
template <int KIND, int D>
struct Step {
  using S = Shape<KIND, D>;
  uint32_t k[S::KT][S::KL * S::KB / 4];   // row 16 t + c: columns of group g
  uint32_t v[S::KT * 4][S::VC * S::VW];   // row 16 t + 4 g + i: columns of lane c
  uint32_t kz[S::NW], vz[S::NW];          // scales of row `lane` (kMx)
};

// the scale bytes of a cache row (D / 32 of them), the first lowest
template <int N>
struct Scales { uint32_t w[(N + 3) / 4]; };
template <int N>
__device__ __forceinline__ Scales<N> row_scales(const uint8_t* p) {
  Scales<N> v;
#pragma unroll
  for (int i = 0; i < (N + 3) / 4; ++i) {
    constexpr int whole = N / 4;
    if (i < whole) {
      v.w[i] = load_raw<uint32_t>(p + 4 * i);
    } else {
      v.w[i] = 0;
      if constexpr (N % 4 >= 2) v.w[i] = load_raw<uint16_t>(p + 4 * i);
      if constexpr (N % 2 == 1) v.w[i] |= (uint32_t)p[N - 1] << (8 * (N % 4 - 1));
    }
  }
  return v;
}

// N words at any multiple of 4 bytes.  ONCE: past the caches.  A long row that
// will not be read again takes no place there (64 sequences of 1 to 8192 keys:
// 110 us a call, 120 without; one of 131072: 54 and 60); rows of short
// segments are often still there from the write (128 sequences of 1 to 300
// keys: 12.4 us a call from the caches, 14.8 past them).
template <int N, bool ONCE>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (N > 4) {
    load_words<4, ONCE>(p, w);
    load_words<N - 4, ONCE>(p + 16, w + 4);
  } else if constexpr (N == 3) {
    load_words<2, ONCE>(p, w);
    load_words<1, ONCE>(p + 8, w + 2);
  } else {
    typedef uint32_t words __attribute__((ext_vector_type(N), aligned(4)));
    const words* src = reinterpret_cast<const words*>(p);
    const words v = ONCE ? __builtin_nontemporal_load(src) : *src;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
  }
}

// WHOLE: a workgroup takes one segment, and there is nothing to join
template <int KIND, int D, bool WHOLE>
__global__ __launch_bounds__(64 * W, (Shape<KIND, D>::PER_CU)) void attn_kernel(const AttnArgs a) {
  using S = Shape<KIND, D>;
  constexpr int KT = S::KT, VC = S::VC, VD = S::VD, ES = S::ES, KEYS = S::KEYS, TILE = S::TILE, KS = S::KS;
  constexpr int NS = S::NS, NW = S::NW;
  constexpr bool WIDE = S::WIDE;
  constexpr int OT = D / 16;                       // output tiles of 16 columns
  constexpr int LP = D + 4;                        // a head's row in LDS: other banks for the next head
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, c = lane & 15, g = lane >> 4;

  const int cap = a.max_pages * a.page, hb_all = a.n_kv * a.blocks;
  int32_t* sums = reinterpret_cast<int32_t*>(lds);  // [n_seq + 1] exclusive sums of the sequences' tiles
  uint32_t u = 0, u_end = 1;
  if constexpr (!WHOLE) {  // (a sequence without keys has one tile)
    __shared__ int32_t wave_sum[W];
    const int per = (a.n_seq + 64 * W - 1) / (64 * W), s0 = tid * per;
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
    if (tid == 64 * W - 1) sums[a.n_seq] = at;
    __syncthreads();
    const uint32_t units = (uint32_t)sums[a.n_seq] * hb_all, runs = min(gridDim.x, units);
    if (blockIdx.x >= runs) return;
    u = run_begin(blockIdx.x, units, runs);
    u_end = run_begin(blockIdx.x + 1, units, runs);
  }

  const int hl = min(16, a.G);               // heads of a block
  float* lds_m = lds + (WHOLE ? 0 : (a.n_seq + 4) & ~3);  // [W][16] m, then l
  float* lds_l = lds_m + W * 16;
  float* lds_o = lds_l + W * 16;              // [W][hl][LP]

  while (u < u_end) {
    int s, hb, nt, tile0 = 0, tile1;
    if constexpr (WHOLE) {
      s = blockIdx.x / (uint32_t)hb_all, hb = blockIdx.x % (uint32_t)hb_all;
      nt = tile1 = max(1, (clampi(a.lens[s], 0, cap) - 1) / TILE + 1);
    } else {
      int lo = 0, hi = a.n_seq - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((uint32_t)sums[mid] * hb_all <= u) lo = mid; else hi = mid - 1;
      }
      s = lo;
      nt = sums[s + 1] - sums[s];
      const uint32_t rem = u - (uint32_t)sums[s] * hb_all;
      hb = rem / (uint32_t)nt, tile0 = rem % (uint32_t)nt;
      tile1 = static_cast<int>(min((uint32_t)nt, tile0 + (u_end - u)));
    }
    const int kv = hb / a.blocks, h0 = kv * a.G + (hb % a.blocks) * 16;
    const int heads = min(16, a.G - (hb % a.blocks) * 16);
    const int len = clampi(a.lens[s], 0, cap);
    const int32_t* table = a.table + (size_t)s * a.max_pages;

    // this lane's part of its head's query: the second operand of S^T
    const char* qr = static_cast<const char*>(a.q) + ((size_t)s * a.n_q + h0 + c) * D * (KIND == 0 ? 4 : 2);
    uint4 q[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      // (WIDE: product i takes columns 64 (i / 2) + 16 g + 8 (i % 2) .. + 8)
      const int at = WIDE ? (i / 2) * 128 + g * 32 + (i % 2) * 16 : i * 64 + g * 16;
      q[i] = c < heads ? *reinterpret_cast<const uint4*>(qr + at) : make_uint4(0, 0, 0, 0);
    }

    float m = -INFINITY, l = 0.f;
    f32x4 o[OT];
#pragma unroll
    for (int i = 0; i < OT; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    // The step's rows are found two steps ahead (a page index from the table),
    // their values are loaded one step ahead, so that memory is never idle
    // while a step is computed.  Loads return in order and are counted, hence
    // none of them stands behind a branch: beyond the last key they read the
    // last one's page entry and row 0, and nothing of them is used.
    auto entry = [&](int key) { return table[page_of(a, (uint32_t)max(min(key, len - 1), 0))]; };
    // cache row of a key (page * n_kv + head) * page_size + slot, ~0 if there is none
    auto row_at = [&](int key, int pg) -> uint32_t {
      const uint32_t off = (uint32_t)key - page_of(a, (uint32_t)key) * a.page;
      return key < len && pg >= 0 && pg < a.n_pages ? ((uint32_t)pg * a.n_kv + kv) * a.page + off : ~0u;
    };
    auto load = [&](uint32_t row, Step<KIND, D>& st) {
      const uint32_t safe = row == ~0u ? 0u : row;
      if constexpr (KIND == kMx) {
        const Scales<NS> kz = row_scales<NS>(a.ks + (size_t)safe * NS), vz = row_scales<NS>(a.vs + (size_t)safe * NS);
#pragma unroll
        for (int i = 0; i < NW; ++i) st.kz[i] = kz.w[i], st.vz[i] = vz.w[i];
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const size_t r = static_cast<uint32_t>(__shfl(static_cast<int>(safe), t * 16 + c, 64));
        const char* p = static_cast<const char*>(a.k) + r * (D * ES) + g * S::KB;
#pragma unroll
        for (int i = 0; i < S::KL; ++i) {
          load_words<S::KB / 4, !WHOLE>(p + i * S::KSTEP, &st.k[t][i * (S::KB / 4)]);
        }
      }
#pragma unroll
      for (int j = 0; j < KT * 4; ++j) {
        const size_t r = static_cast<uint32_t>(__shfl(static_cast<int>(safe), (j >> 2) * 16 + g * 4 + (j & 3), 64));
#pragma unroll
        for (int part = 0; part < VC; ++part) {
          const char* p = static_cast<const char*>(a.v) + r * (D * ES) + (part * (D / 2) + c * VD) * ES;
          if constexpr (VD * ES % 4 == 0) {
            load_words<S::VW, !WHOLE>(p, &st.v[j][part * S::VW]);
          } else {  // 2 or 6 bytes
            if constexpr (S::VW == 2) st.v[j][part * 2] = load_raw<uint32_t>(p);
            st.v[j][part * S::VW + S::VW - 1] = load_raw<uint16_t>(p + (S::VW - 1) * 4);
          }
        }
      }
    };
    auto compute = [&](uint32_t row, const Step<KIND, D>& st) {
      const uint32_t there = static_cast<uint32_t>(__ballot(row != ~0u));  // bit j: key j of the step (lanes repeat)
      // S^T = K Q^T
      f32x4 sc[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (KIND == kMx) {
          uint32_t z[NW];
#pragma unroll
          for (int i = 0; i < NW; ++i) z[i] = static_cast<uint32_t>(__shfl(static_cast<int>(st.kz[i]), t * 16 + c, 64));
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            // the block of product i's columns of this lane (WIDE: i and i + 1 lie in one word)
            const int blk = WIDE ? i / 2 * 2 + g / 2 : i;
            const float f = mx_scale((z[i / 4] >> (8 * (blk & 3))) & 255u);
            const uint32_t lo = st.k[t][2 * i], hi = st.k[t][2 * i + 1];
            const bf16x2_t k0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false);
            const bf16x2_t k1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true);
            const bf16x2_t k2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false);
            const bf16x2_t k3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true);
            const bf16x8 ka = {k0[0], k0[1], k1[0], k1[1], k2[0], k2[1], k3[0], k3[1]};
            sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, __builtin_bit_cast(bf16x8, q[i]), sc[t], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            if constexpr (KIND == 1) {
              const u32x4 kk = {st.k[t][4 * i], st.k[t][4 * i + 1], st.k[t][4 * i + 2], st.k[t][4 * i + 3]};
              sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk),
                                                              __builtin_bit_cast(bf16x8, q[i]), sc[t], 0, 0, 0);
            } else {
              const uint32_t qa[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
              for (int e = 0; e < 4; ++e)
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(st.k[t][4 * i + e]), __uint_as_float(qa[e]),
                                                             sc[t], 0, 0, 0);
            }
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
          const float p = __builtin_amdgcn_exp2f(sc[t][i] - ref);
          sc[t][i] = p;
          sum += p;
        }
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      l *= keep;
#pragma unroll
      for (int i = 0; i < OT; ++i) o[i] *= keep;
      l += sum;
      m = top;

      // O^T += V^T P^T: the keys of a product in the order 16 t + 4 g + i.
      // A row that is not there has weight 0 and is taken as 0 (it may hold NaN).
      uint32_t ok[KT * 4];
#pragma unroll
      for (int j = 0; j < KT * 4; ++j) ok[j] = (there >> ((j >> 2) * 16 + g * 4 + (j & 3))) & 1u ? ~0u : 0u;
#pragma unroll
      for (int part = 0; part < VC; ++part) {
        if constexpr (KIND == 0) {
#pragma unroll
          for (int e = 0; e < VD; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[part * VD + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __uint_as_float(st.v[j][part * S::VW + e] & ok[j]), sc[0][j], o[part * VD + e], 0, 0, 0);
        } else {
          const int col = part * (D / 2) + c * VD;  // this lane's first column of the part
          // the weights in two bf16 parts, a product each: what the first leaves of
          // a weight (2^-8 of it at most, exact in float32) is rounded to 2^-16 of it
          u32x4 pw, pr;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p0 = sc[j < 2 ? 0 : KT - 1][2 * (j & 1)], p1 = sc[j < 2 ? 0 : KT - 1][2 * (j & 1) + 1];
            const uint32_t w = pack_bf16x2(p0, p1);
            pw[j] = w;
            pr[j] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
          }
          const bf16x8 pb = __builtin_bit_cast(bf16x8, pw), pl = __builtin_bit_cast(bf16x8, pr);
          uint32_t vv[8][VD / 2];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if constexpr (KIND == 1) {
#pragma unroll
              for (int e = 0; e < VD / 2; ++e) vv[j][e] = st.v[j][part * S::VW + e] & ok[j];
            } else {
              uint32_t z[NW];
#pragma unroll
              for (int i = 0; i < NW; ++i)
                z[i] = static_cast<uint32_t>(__shfl(static_cast<int>(st.vz[i]), (j >> 2) * 16 + g * 4 + (j & 3), 64));
              auto scale_at = [&](int x) {  // of column x
                const uint32_t word = NW > 1 && x >= 128 ? z[NW - 1] : z[0];
                return mx_scale((word >> (x / 32 % 4 * 8)) & 255u);
              };
              const float f0 = scale_at(col);
#pragma unroll
              for (int e = 0; e < VD / 2; ++e) {
                // a lane's six columns may lie in two blocks of 32
                const float f = VD == 6 ? scale_at(col + 2 * e) : f0;
                const uint32_t raw = st.v[j][part * S::VW + e / 2];
                const bf16x2_t w = e % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, f, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, f, false);
                vv[j][e] = __builtin_bit_cast(uint32_t, w) & ok[j];
              }
            }
          }
#pragma unroll
          for (int e = 0; e < VD / 2; ++e) {
            u32x4 lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              lo[j] = __builtin_amdgcn_perm(vv[2 * j + 1][e], vv[2 * j][e], 0x05040100u);
              hi[j] = __builtin_amdgcn_perm(vv[2 * j + 1][e], vv[2 * j][e], 0x07060302u);
            }
            const int x = part * VD + 2 * e;
            const bf16x8 v0 = __builtin_bit_cast(bf16x8, lo), v1 = __builtin_bit_cast(bf16x8, hi);
            o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pb, o[x], 0, 0, 0);
            o[x + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pb, o[x + 1], 0, 0, 0);
            o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pl, o[x], 0, 0, 0);
            o[x + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pl, o[x + 1], 0, 0, 0);
          }
        }
      }
    };
    {
      int key = tile0 * TILE + wv * KEYS + (lane & (KEYS - 1));  // this lane's key of the step
      uint32_t row = row_at(key, entry(key));
      int pg = entry(key + TILE);
      Step<KIND, D> even, odd;
      load(row, even);
      int left = tile1 - tile0;
      for (; left > 2; left -= 2, key += 2 * TILE) {
        const uint32_t row1 = row_at(key + TILE, pg);
        pg = entry(key + 2 * TILE);
        load(row1, odd);
        compute(row, even);
        row = row_at(key + 2 * TILE, pg);
        pg = entry(key + 3 * TILE);
        load(row, even);
        compute(row1, odd);
      }
      if (left == 2) {
        const uint32_t row1 = row_at(key + TILE, pg);
        load(row1, odd);
        compute(row, even);
        compute(row1, odd);
      } else {
        compute(row, even);
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
    for (int w = 1; w < W; ++w) top = fmaxf(top, lds_m[w * 16 + c]);
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    if (c < heads)
#pragma unroll
      for (int x = 0; x < OT; x += 2)  // (VD is even)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float2*>(lds_o + (wv * hl + c) * LP + (x / VD) * (D / 2) + (4 * g + i) * VD + x % VD) =
              make_float2(o[x][i] * f, o[x + 1][i] * f);
    __syncthreads();
    const bool first = tile0 == 0, end = tile1 == nt;
    if (!WHOLE && tid == 0) {  // which runs share the segment
      int32_t* of = a.shared + 2 * ((size_t)s * hb_all + hb);
      if (first) of[0] = blockIdx.x;
      if (end) of[1] = blockIdx.x;
    }
    const size_t slot = 2 * (size_t)blockIdx.x + (first ? 1 : 0);  // of a partial result
    for (int i = tid; i < heads * D; i += 64 * W) {
      const int h = i / D;
      float top = lds_m[h];
#pragma unroll
      for (int w = 1; w < W; ++w) top = fmaxf(top, lds_m[w * 16 + h]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, v = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        sum += lds_l[w * 16 + h] * __builtin_amdgcn_exp2f(lds_m[w * 16 + h] - ref);
        v += lds_o[(w * hl + h) * LP + i - h * D];
      }
      if (WHOLE || (first && end)) {
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
    if constexpr (WHOLE) return;
    u += tile1 - tile0;
  }
}

// The partial results of the segments that several runs share, in order; a
// workgroup a (segment, head).  The weights 2^(m - top) of the parts are formed
// once, then groups of D / 4 lanes take the parts in turn.
template <bool BF16>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs a, int D) {
  __shared__ float weight[kRuns];
  __shared__ float red[2][4];
  __shared__ float4 acc[256];
  const int hb_all = a.n_kv * a.blocks;
  const int seg = blockIdx.x, h = blockIdx.y, s = seg / hb_all, hb = seg % hb_all;
  const int r0 = a.shared[2 * (size_t)seg], parts = a.shared[2 * (size_t)seg + 1] - r0 + 1;
  if (parts == 1 || h >= min(16, a.G - (hb % a.blocks) * 16)) return;  // one run wrote the output
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  auto slot = [&](int i) -> size_t { return 2 * (size_t)(r0 + i) + (i == 0 ? 1 : 0); };
  float top = -INFINITY;
  for (int i = tid; i < parts; i += 256) {
    const float m = a.part[slot(i) * 32 + h];
    weight[i] = m;
    top = fmaxf(top, m);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if (lane == 0) red[0][wv] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < parts; i += 256) {
    const float w = __builtin_amdgcn_exp2f(weight[i] - ref);
    weight[i] = w;
    sum = fmaf(a.part[slot(i) * 32 + 16 + h], w, sum);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) red[1][wv] = sum;
  __syncthreads();
  sum = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const int cols = D / 4, groups = 256 / cols, c = tid % cols, g = tid / cols;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (g < groups) {
    auto add = [&](int i) {
      const float4 o = *reinterpret_cast<const float4*>(a.part_o + (slot(i) * 16 + h) * D + 4 * c);
      const float w = weight[i];
      v.x = fmaf(o.x, w, v.x), v.y = fmaf(o.y, w, v.y), v.z = fmaf(o.z, w, v.z), v.w = fmaf(o.w, w, v.w);
    };
    int i = g;
    for (; i + 3 * groups < parts; i += 4 * groups) {
      add(i);
      add(i + groups);
      add(i + 2 * groups);
      add(i + 3 * groups);
    }
    for (; i < parts; i += groups) add(i);
    acc[g * cols + c] = v;
  }
  __syncthreads();
  if (tid >= cols) return;
  v = acc[tid];
  for (int k = 1; k < min(groups, parts); ++k) {
    const float4 o = acc[k * cols + tid];
    v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
  }
  // no weight at all: zeros, whatever stands in v (0 times an infinity is NaN)
  if (sum == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
  const float r = sum == 0.f ? 0.f : 1.f / sum;
  const size_t at = ((size_t)s * a.n_q + (hb / a.blocks) * a.G + (hb % a.blocks) * 16 + h) * D + 4 * tid;
  if constexpr (BF16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) =
        make_uint2(pack_bf16x2(v.x * r, v.y * r), pack_bf16x2(v.z * r, v.w * r));
  else
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v.x * r, v.y * r, v.z * r, v.w * r);
}

template <int KIND, int D>
hipError_t launch_d(const AttnArgs& a, int max_keys, hipStream_t s) {
  using S = Shape<KIND, D>;
  const long long segments = (long long)a.n_seq * a.n_kv * a.blocks, tiles = std::max(1, (max_keys - 1) / S::TILE + 1);
  const size_t lds = ((size_t)2 * W * 16 + (size_t)W * std::min(a.G, 16) * (D + 4)) * 4;
  // Few keys: a workgroup for each segment.  One alone takes 4 us and 1.1 us a
  // tile (D 128), the runs' start and join about 8 us, so up to five tiles (D >
  // 128: two), and where the segments fill half the card (128) up to 16.  Long
  // rows (D > 128, or more than 256 bytes) stop at eight there until the segments
  // fill all of it (256).  Whole against runs, us, 4 key/value heads: 1 sequence of
  // 515 keys, 5 tiles 9.2 / 11.6, of 1024, 8 tiles 12.4 / 11.6; 64 of 1 to 1024 16 /
  // 25, to 2048, 16 tiles 34 / 38; float32, D 64, 8 heads, 8 of 1 to 515, 9 tiles
  // 12.6 / 11.8; D 256: 1 of 515 17 / 14, 64 of 1 to 1024 37 / 50.  Long rows, 128
  // segments, of 8, 9 and 16 tiles: D 256 27 / 31, 31 / 32, 54 / 39, in 8 bits 22 /
  // 28, 24 / 29, 37 / 37, float32, D 128 21 / 20, 22 / 21, 37 / 27; 256 segments of
  // 16 tiles: 65 / 68, 42 / 60, 42 / 45
  constexpr bool LONG = D > 128 || D * S::ES > 256;
  if (tiles <= (D > 128 ? 2 : 5) || (segments >= 128 && tiles <= (LONG && segments < 256 ? 8 : 16))) {
    attn_kernel<KIND, D, true><<<(unsigned)segments, 64 * W, lds, s>>>(a);
    return hipGetLastError();
  }
  // runs that are resident at once, so that all of them start together and end
  // together (64 sequences of up to 8192 keys, D 128: 256 / 512 / 1024 runs 135 /
  // 120 / 124 us; 8 sequences, D 256: 43 / 50 / 61)
  const int grid = (int)std::min<long long>(256 * S::PER_CU, tiles * segments);
  attn_kernel<KIND, D, false><<<grid, 64 * W, lds + ((a.n_seq + 4) & ~3) * 4, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  attn_join_kernel<KIND != 0><<<dim3((unsigned)segments, std::min(a.G, 16)), 256, 0, s>>>(a, D);
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
  if (n_seq > kMaxSeq || max_keys > (1 << 30)) return false;
  const long long blocks = (n_q / n_kv + 15) / 16;
  const long long segments = (long long)n_seq * n_kv * blocks;
  // (a launch counts its threads, 256 a segment, in 32 bits)
  return segments <= 1 << 23 && (long long)((max_keys - 1) / 64 + 1) <= INT32_MAX / std::max(1LL, segments);
}

size_t attn_ws_bytes(int n_seq, int n_q, int n_kv, int D, int max_keys) {
  (void)max_keys;
  const size_t segments = (size_t)n_seq * n_kv * ((n_q / n_kv + 15) / 16);
  return up256(segments * 8) + up256((size_t)2 * kRuns * 32 * 4) + (size_t)2 * kRuns * 16 * D * 4;
}

hipError_t launch_attn_decode(const void* q, int kind, int n_seq, int n_q, int n_kv, int D, const void* k_cache,
                              const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int n_pages,
                              int page_size, const int32_t* block_table, int max_pages, const int32_t* lens,
                              float scale, void* out, void* ws, hipStream_t s) {
  char* w = static_cast<char*>(ws);
  AttnArgs a{};
  a.q = q, a.k = k_cache, a.v = v_cache, a.ks = k_scale, a.vs = v_scale;
  a.table = block_table, a.lens = lens, a.out = out;
  a.shared = reinterpret_cast<int32_t*>(w);
  a.part = reinterpret_cast<float*>(w + up256((size_t)n_seq * n_kv * ((n_q / n_kv + 15) / 16) * 8));
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
