// Page tables and slot maps from request lengths.
//
//   need(s) = ceil((len + add) / page) - ceil(len / page)
//
// One workgroup walks the sequences 1024 at a time: finished ones push their
// pages on the stack of free ones, then exclusive sums over the sequences
// place every request's rows and pages, and the new pages are copied from the
// top of the stack.  The work is a few dependent loads and scans, so latency
// bounds it.  The slot map of many rows is a second launch over the rows.
#include "block.hpp"

namespace decomoe {
namespace {

constexpr int KX = 1024;  // sequences a pass
// rows up to which the one workgroup also writes the slot map
constexpr int KV_ROWS_ONE = 8192;

// inclusive sum over the workgroup's KX threads; tmp: KX / 64 values
template <typename T>
__device__ __forceinline__ T scan_wg(T v, T* tmp) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  __syncthreads();  // tmp of an earlier scan has been read
  if (lane == 63) tmp[wv] = v;
  __syncthreads();
  T before = 0;
  for (int w = 0; w < wv; ++w) before += tmp[w];
  return v + before;
}

// the first entry s of up[0, n) with up[s] > i (i < up[n - 1])
__device__ __forceinline__ int first_above(const int32_t* up, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (up[mid] > i) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ int slot_of(const int32_t* row, int pos, int page, int n_pages) {
  const int p = row[pos / page];
  return p >= 0 && p < n_pages ? p * page + pos % page : -1;
}

__global__ __launch_bounds__(KX) void kv_extend_kernel(
    const int32_t* len_in, const int32_t* __restrict__ add, int n_seq, int page, int max_pages, int n_pages,
    int rows_max, const int32_t* n_free_in, int32_t* __restrict__ table, int32_t* __restrict__ free_pages,
    int32_t* len_out, int32_t* n_free_out, int32_t* __restrict__ row_offsets, int32_t* __restrict__ slot_map,
    int32_t* __restrict__ positions, int32_t* __restrict__ accepted, int32_t* __restrict__ status, int write_rows) {
  __shared__ long long tmp[KX / 64];
  __shared__ int32_t upto[KX], first[KX], base[KX], rows_to[KX];
  const int tid = threadIdx.x;
  const int cap = max_pages * page;
  const int n_free = clampi(*n_free_in, 0, n_pages);
  auto length = [&](int s) { return clampi(len_in[s], 0, cap); };
  auto pages = [&](int len) { return len > 0 ? (len - 1) / page + 1 : 0; };

  // finished sequences: their pages on top of the stack
  int given = 0;
  for (int s0 = 0; s0 < n_seq; s0 += KX) {
    const int s = s0 + tid, in = min(KX, n_seq - s0);
    const bool gone = s < n_seq && add[s] < 0;
    if (!__syncthreads_or(gone)) continue;
    const int have = gone ? pages(length(s)) : 0;
    const int up = static_cast<int>(scan_wg<long long>(have, tmp));
    upto[tid] = up;
    base[tid] = up - have;
    __syncthreads();
    const int all = upto[in - 1];
    for (int i = tid; i < all; i += KX) {
      const int k = first_above(upto, in, i);
      const long long at = (long long)n_free + given + i;
      if (at < n_pages) free_pages[at] = table[(size_t)(s0 + k) * max_pages + (i - base[k])];
    }
    given += all;
    __syncthreads();
  }
  const int avail = static_cast<int>(min((long long)n_pages, (long long)n_free + given));

  // the others, in order
  long long rows = 0, needed = 0;
  int taken = 0, refused = 0;
  for (int s0 = 0; s0 < n_seq; s0 += KX) {
    const int s = s0 + tid, in = min(KX, n_seq - s0);
    const bool live = s < n_seq;
    const int want = live ? add[s] : 0, len = live ? length(s) : 0;
    const bool gone = want < 0;
    const int fresh = gone ? 0 : want;
    const long long row_end = rows + scan_wg<long long>(fresh, tmp);
    const bool fits = live && !gone && (long long)len + fresh <= cap && row_end <= rows_max;
    const int have = pages(len);
    const int need = fits ? pages(len + fresh) - have : 0;
    const long long need_end = needed + scan_wg<long long>(need, tmp);
    const bool served = fits && (need == 0 || need_end <= avail);
    const int take = served ? need : 0;
    // pages taken: those of the served ones are the first of all needed
    const int up = static_cast<int>(scan_wg<long long>(take, tmp));
    upto[tid] = up;
    first[tid] = have - (up - take);  // table column of page i of this pass: i + first
    if (live) {
      len_out[s] = gone ? 0 : served ? len + fresh : len;
      accepted[s] = gone || served ? 1 : 0;
      row_offsets[s + 1] = static_cast<int32_t>(min(row_end, (long long)rows_max));
    }
    base[tid] = served ? len : -1;
    rows_to[tid] = static_cast<int32_t>(min(row_end, (long long)rows_max));
    refused += __syncthreads_count(live && !gone && !served);
    const int all = upto[in - 1];
    for (int i = tid; i < all; i += KX) {
      const int k = first_above(upto, in, i);
      table[(size_t)(s0 + k) * max_pages + (i + first[k])] = free_pages[avail - 1 - taken - i];
    }
    const int row0 = static_cast<int>(min(rows, (long long)rows_max)), row1 = rows_to[in - 1];
    if (tid == KX - 1) {
      tmp[0] = row_end;
      tmp[1] = need_end;
    }
    __syncthreads();  // the new table entries are visible to the workgroup
    rows = tmp[0];
    needed = tmp[1];
    if (write_rows)
      for (int r = row0 + tid; r < row1; r += KX) {
        const int k = first_above(rows_to, in, r);
        const int pos = base[k] + r - (k ? rows_to[k - 1] : row0);
        const int slot = base[k] >= 0 ? slot_of(table + (size_t)(s0 + k) * max_pages, pos, page, n_pages) : -1;
        slot_map[r] = slot;
        positions[r] = slot >= 0 ? pos : 0;
      }
    taken += all;
    __syncthreads();  // the arrays of this pass have been read
  }
  const int end = static_cast<int>(min(rows, (long long)rows_max));
  if (write_rows)
    for (int r = end + tid; r < rows_max; r += KX) {
      slot_map[r] = -1;
      positions[r] = 0;
    }
  if (tid == 0) {
    row_offsets[0] = 0;
    *n_free_out = avail - taken;
    status[0] = end;
    status[1] = taken;
    status[2] = refused;
    status[3] = avail - n_free;
  }
}

// slot_map and positions of many rows, after kv_extend_kernel
__global__ __launch_bounds__(256) void kv_rows_kernel(const int32_t* __restrict__ add, int n_seq, int page,
                                                      int max_pages, int n_pages, int rows_max,
                                                      const int32_t* __restrict__ table,
                                                      const int32_t* __restrict__ len_out,
                                                      const int32_t* __restrict__ row_offsets,
                                                      const int32_t* __restrict__ accepted,
                                                      int32_t* __restrict__ slot_map,
                                                      int32_t* __restrict__ positions) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= rows_max) return;
  int slot = -1, pos = 0;
  if (n_seq > 0 && r < row_offsets[n_seq]) {
    const int s = first_above(row_offsets + 1, n_seq, r);
    if (accepted[s]) {
      pos = len_out[s] - add[s] + (r - row_offsets[s]);
      slot = slot_of(table + (size_t)s * max_pages, pos, page, n_pages);
    }
  }
  slot_map[r] = slot;
  positions[r] = slot >= 0 ? pos : 0;
}

}  // namespace

hipError_t launch_kv_extend(const int32_t* len_in, const int32_t* add, int n_seq, int page_size, int max_pages,
                            int n_pages, int rows_max, const int32_t* n_free_in, int32_t* block_table,
                            int32_t* free_pages, int32_t* len_out, int32_t* n_free_out, int32_t* row_offsets,
                            int32_t* slot_map, int32_t* positions, int32_t* accepted, int32_t* status,
                            hipStream_t s) {
  const bool one = rows_max <= KV_ROWS_ONE;
  kv_extend_kernel<<<1, KX, 0, s>>>(len_in, add, n_seq, page_size, max_pages, n_pages, rows_max, n_free_in,
                                    block_table, free_pages, len_out, n_free_out, row_offsets, slot_map, positions,
                                    accepted, status, one ? 1 : 0);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  kv_rows_kernel<<<(rows_max + 255) / 256, 256, 0, s>>>(add, n_seq, page_size, max_pages, n_pages, rows_max,
                                                        block_table, len_out, row_offsets, accepted, slot_map,
                                                        positions);
  return hipGetLastError();
}

}  // namespace decomoe
