// Page tables and slot maps from request lengths.
//
//   need(s) = ceil((len + add) / page) - ceil(len / page)
//
// One workgroup walks the sequences: finished ones push their pages on the
// stack of free ones, then exclusive sums over the others place every
// request's rows and pages.  A row's slot follows from those sums alone (the
// n-th page taken is the n-th from the top of the stack), and the row that
// begins a page writes its table entry, so the rows need no order.  Few rows
// are done by the same workgroup, many by a second launch that forms the sums
// of its own part again.  All of it is a few dependent loads and scans:
// latency bounds it (64 sequences, a token each: 4.3 us; 256 sequences, 230
// thousand rows, 14 thousand pages taken and 6 thousand given back: 11.8 and
// 7.9 us in the two launches).
#include "block.hpp"

namespace decomoe {
namespace {

// rows up to which the one workgroup also writes the slot map (4, 64, 200
// sequences, us in one launch and in two: 2048 rows 9.4, 11.5, 8.9 and 11.8,
// 13.8, 12.0; 4096 rows 14.7, 16.8, 17.1 and 12.0, 14.1, 14.5)
constexpr int KV_ROWS_ONE = 2048;
constexpr int KV_ROWS = 1024;  // rows of a workgroup of the second launch

// inclusive sum over the workgroup's threads; tmp: a value a wavefront
template <typename T, int THREADS>
__device__ __forceinline__ T scan_wg(T v, T* tmp) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  if constexpr (THREADS > 64) {
    constexpr int WAVES = THREADS / 64;
    __syncthreads();  // tmp of an earlier scan has been read
    if (lane == 63) tmp[wv] = v;
    __syncthreads();
    T w = lane < WAVES ? tmp[lane] : 0;  // the sums of the wavefronts before
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) {
      const T u = __shfl_up(w, o, 64);
      if (lane >= o) w += u;
    }
    const T before = __shfl(w, max(wv - 1, 0), 64);
    if (wv) v += before;
  }
  return v;
}

// for each i[j] the first entry s of the N (a power of two) ascending ones with
// up[s] > i[j] (i < up[N - 1]); the J searches' reads are in flight together
template <int N, int J>
__device__ __forceinline__ void first_above(const int32_t* up, const int (&i)[J], int (&s)[J]) {
#pragma unroll
  for (int j = 0; j < J; ++j) s[j] = 0;
#pragma unroll
  for (int b = N / 2; b >= 1; b >>= 1)
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (up[s[j] + b - 1] <= i[j]) s[j] += b;
}

__device__ __forceinline__ int pages_of(int len, int page) { return len > 0 ? (len - 1) / page + 1 : 0; }

// one row: token `pos` of a sequence that held `len` and whose first new page
// is the `nth` taken (top: entries of the stack before any was taken)
__device__ __forceinline__ void place_row(int r, bool served, int pos, int len, int nth, int top, int page, int n_pages,
                                          int32_t* table_row, const int32_t* free_pages, int32_t* slot_map,
                                          int32_t* positions) {
  int slot = -1;
  if (served) {
    const int at = pos / page, off = pos - at * page, have = pages_of(len, page);
    int p;
    if (at < have) {
      p = table_row[at];
    } else {
      p = free_pages[top - 1 - (nth + at - have)];
      if (off == 0) table_row[at] = p;
    }
    if (p >= 0 && p < n_pages) slot = p * page + off;
  }
  slot_map[r] = slot;
  positions[r] = slot >= 0 ? pos : 0;
}

// KX sequences a pass
template <int KX>
__global__ __launch_bounds__(KX) void kv_extend_kernel(
    const int32_t* len_in, const int32_t* __restrict__ add, int n_seq, int page, int max_pages, int n_pages,
    int rows_max, const int32_t* n_free_in, int32_t* table, int32_t* free_pages, int32_t* len_out,
    int32_t* n_free_out, int32_t* __restrict__ row_offsets, int32_t* __restrict__ slot_map,
    int32_t* __restrict__ positions, int32_t* __restrict__ accepted, int32_t* __restrict__ status, int write_rows) {
  __shared__ long long tmp[KX / 64];
  __shared__ int tmp32[KX / 64];
  __shared__ int32_t upto[KX], base[KX], nth[KX];
  __shared__ long long carry[2];
  __shared__ int last_page;
  const int tid = threadIdx.x;
  const int cap = max_pages * page;
  // the first pass's sequence, before anything waits
  const int n_free = clampi(*n_free_in, 0, n_pages);
  int want = tid < n_seq ? add[tid] : 0;
  int len = tid < n_seq ? clampi(len_in[tid], 0, cap) : 0;

  // finished sequences: their pages on top of the stack
  int given = 0;
  for (int s0 = 0; s0 < n_seq; s0 += KX) {
    const int s = s0 + tid;
    const int w = s0 ? (s < n_seq ? add[s] : 0) : want;
    if (!__syncthreads_or(w < 0)) continue;
    const int have = w < 0 ? pages_of(s0 ? clampi(len_in[s], 0, cap) : len, page) : 0;
    const int up = scan_wg<int, KX>(have, tmp32);
    upto[tid] = up;
    base[tid] = up - have;
    __syncthreads();
    const int all = upto[KX - 1];
    for (int i0 = tid; i0 < all; i0 += 4 * KX) {  // four copies in flight
      int v[4], at[4], k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j] = min(i0 + j * KX, all - 1);
      first_above<KX>(upto, at, k);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = table[(size_t)(s0 + k[j]) * max_pages + (at[j] - base[k[j]])];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * KX;
        const long long at = (long long)n_free + given + i;
        if (i < all && at < n_pages) free_pages[at] = v[j];
      }
    }
    given += all;
    __syncthreads();  // the arrays have been read, the stack is written
  }
  const int top = static_cast<int>(min((long long)n_pages, (long long)n_free + given));

  // the others, in order
  long long rows = 0;
  int needed = 0, taken = 0, refused = 0;
  for (int s0 = 0; s0 < n_seq; s0 += KX) {
    const int s = s0 + tid;
    const bool live = s < n_seq;
    if (s0) {
      want = live ? add[s] : 0;
      len = live ? clampi(len_in[s], 0, cap) : 0;
    }
    const bool gone = want < 0;
    const int fresh = gone ? 0 : want;
    const long long row_end = rows + scan_wg<long long, KX>(fresh, tmp);
    const bool fits = live && !gone && (long long)len + fresh <= cap && row_end <= rows_max;
    const int need = fits ? pages_of(len + fresh, page) - pages_of(len, page) : 0;
    const int need_end = needed + scan_wg<int, KX>(need, tmp32);
    // the pages needed up to a served sequence are all taken: what is refused
    // for want of pages comes behind it
    const bool served = fits && (need == 0 || need_end <= top);
    const int end = static_cast<int>(min(row_end, (long long)rows_max));
    if (live) {
      len_out[s] = gone ? 0 : served ? len + fresh : len;
      accepted[s] = gone || served ? 1 : 0;
      row_offsets[s + 1] = end;
    }
    if (tid == 0) last_page = taken;
    if (tid == KX - 1) carry[0] = row_end, carry[1] = need_end;
    refused += __syncthreads_count(live && !gone && !served);
    if (served && need) atomicMax(&last_page, need_end);  // (whole numbers: any order)
    if (write_rows) {
      if (!__syncthreads_or(fresh > 1)) {  // a token each at the most: every thread its own row
        if (fresh && row_end <= rows_max)
          place_row(end - 1, served, len, len, need_end - need, top, page, n_pages, table + (size_t)s * max_pages,
                    free_pages, slot_map, positions);
      } else {
        upto[tid] = end;
        base[tid] = served ? len : -1;
        nth[tid] = need_end - need;
        __syncthreads();
        const int row0 = static_cast<int>(min(rows, (long long)rows_max)), row1 = upto[KX - 1];
        for (int r = row0 + tid; r < row1; r += KX) {
          int at[1] = {r}, ks[1];
          first_above<KX>(upto, at, ks);
          const int k = ks[0], b = base[k];
          place_row(r, b >= 0, b + r - (k ? upto[k - 1] : row0), b, nth[k], top, page, n_pages,
                    table + (size_t)(s0 + k) * max_pages, free_pages, slot_map, positions);
        }
      }
    }
    __syncthreads();
    rows = carry[0];
    needed = static_cast<int>(carry[1]);
    taken = last_page;
    __syncthreads();  // this pass's arrays have been read
  }
  const int end = static_cast<int>(min(rows, (long long)rows_max));
  if (write_rows)
    for (int r = end + tid; r < rows_max; r += KX) {
      slot_map[r] = -1;
      positions[r] = 0;
    }
  if (tid == 0) {
    row_offsets[0] = 0;
    *n_free_out = top - taken;
    status[0] = end;
    status[1] = taken;
    status[2] = refused;
    status[3] = top - n_free;
  }
}

// slot_map, positions and table entries of many rows, after kv_extend_kernel:
// lengths before the step and the order of the pages follow from its outputs
__global__ __launch_bounds__(256) void kv_rows_kernel(const int32_t* __restrict__ add, int n_seq, int page,
                                                      int max_pages, int n_pages, int rows_max, int32_t* table,
                                                      const int32_t* __restrict__ free_pages,
                                                      const int32_t* __restrict__ len_out,
                                                      const int32_t* __restrict__ n_free_out,
                                                      const int32_t* __restrict__ row_offsets,
                                                      const int32_t* __restrict__ accepted,
                                                      const int32_t* __restrict__ status,
                                                      int32_t* __restrict__ slot_map,
                                                      int32_t* __restrict__ positions) {
  __shared__ int tmp[4];
  __shared__ int32_t upto[256], base[256], nth[256];
  const int tid = threadIdx.x;
  const int r0 = blockIdx.x * KV_ROWS, r_end = min(rows_max, r0 + KV_ROWS);
  const int total = n_seq ? row_offsets[n_seq] : 0;
  const int top = *n_free_out + status[1];
  const int r1 = min(r_end, total);
  if (r0 < r1) {
    auto need_of = [&](int s) {
      const int a = add[s], l = len_out[s];
      return a > 0 && accepted[s] ? pages_of(l, page) - pages_of(l - a, page) : 0;
    };
    // sequences [s0, s1] hold these rows; pages taken by the ones before s0.  All
    // sequences are looked at: independent loads, where a search would wait for
    // each of its own
    int c0s = 0, c1s = 0, before = 0;
    for (int s = tid; s < n_seq; s += 256) {
      const int e = row_offsets[s + 1], need = need_of(s);
      c0s += e <= r0;
      c1s += e <= r1 - 1;
      before += e <= r0 ? need : 0;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      c0s += __shfl_xor(c0s, o, 64);
      c1s += __shfl_xor(c1s, o, 64);
      before += __shfl_xor(before, o, 64);
    }
    if ((tid & 63) == 0) upto[tid >> 6] = c0s, base[tid >> 6] = c1s, nth[tid >> 6] = before;
    __syncthreads();
    const int s0 = upto[0] + upto[1] + upto[2] + upto[3], s1 = base[0] + base[1] + base[2] + base[3];
    int taken = nth[0] + nth[1] + nth[2] + nth[3];
    for (int c0 = s0; c0 <= s1; c0 += 256) {
      const int s = c0 + tid;
      const bool live = s <= s1;
      const int need = live ? need_of(s) : 0;
      const int up = scan_wg<int, 256>(need, tmp);
      __syncthreads();  // the arrays have been read
      upto[tid] = live ? row_offsets[s + 1] : INT32_MAX;
      base[tid] = live && accepted[s] && add[s] >= 0 ? len_out[s] - add[s] : -1;
      nth[tid] = taken + up - need;
      if (tid == 255) tmp[0] = up;
      __syncthreads();
      const int begin = row_offsets[c0], lo = max(r0, begin), hi = min(r1, upto[255]);
      for (int r = lo + tid; r < hi; r += 256) {
        int at[1] = {r}, ks[1];
        first_above<256>(upto, at, ks);
        const int k = ks[0], b = base[k];
        place_row(r, b >= 0, b + r - (k ? upto[k - 1] : begin), b, nth[k], top, page, n_pages,
                  table + (size_t)(c0 + k) * max_pages, free_pages, slot_map, positions);
      }
      taken += tmp[0];
    }
  }
  for (int r = max(r0, total) + tid; r < r_end; r += 256) {
    slot_map[r] = -1;
    positions[r] = 0;
  }
}

}  // namespace

hipError_t launch_kv_extend(const int32_t* len_in, const int32_t* add, int n_seq, int page_size, int max_pages,
                            int n_pages, int rows_max, const int32_t* n_free_in, int32_t* block_table,
                            int32_t* free_pages, int32_t* len_out, int32_t* n_free_out, int32_t* row_offsets,
                            int32_t* slot_map, int32_t* positions, int32_t* accepted, int32_t* status,
                            hipStream_t s) {
  const bool one = rows_max <= KV_ROWS_ONE;
#define EXTEND(KX)                                                                                                   \
  kv_extend_kernel<KX><<<1, KX, 0, s>>>(len_in, add, n_seq, page_size, max_pages, n_pages, rows_max, n_free_in,      \
                                        block_table, free_pages, len_out, n_free_out, row_offsets, slot_map,         \
                                        positions, accepted, status, one ? 1 : 0)
  if (n_seq <= 256 && one) EXTEND(256);
  else EXTEND(1024);
#undef EXTEND
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  kv_rows_kernel<<<(rows_max - 1) / KV_ROWS + 1, 256, 0, s>>>(add, n_seq, page_size, max_pages, n_pages, rows_max,
                                                            block_table, free_pages, len_out, n_free_out, row_offsets,
                                                            accepted, status, slot_map, positions);
  return hipGetLastError();
}

}  // namespace decomoe
