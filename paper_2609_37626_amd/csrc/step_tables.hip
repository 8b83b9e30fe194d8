// gfx950 kernel of splash_step_tables: a step's pages, slots and positions from
// the requests' lengths.
//
// Two sums run over the requests, of new tokens and of new pages.  Every
// workgroup forms both itself (a request or a few per thread, then a scan over
// the workgroup), keeps them in LDS, and fills a slice of the step's rows, whose
// requests it finds by bisection: one launch and nothing to wait for between
// workgroups.  The row of a page's first token writes that page's table entry;
// an entry that the step adds is computed from the free list wherever it is
// needed and never read back from the table.
//
// Bound: latency (lengths, scan, list entry, store, one after the other).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "step.hpp"

namespace splash {

namespace {

constexpr int kThreads = 1024;
constexpr int kRowsPerGroup = kThreads;  // (131,072 rows: 5.4 us, with 4,096 rows a workgroup 8.8)
constexpr int kPerThread = kMaxTableBatch / kThreads;

struct Lens {
  int32_t seq, fresh;  // tokens after the step, and the new ones among them
};
__device__ __forceinline__ Lens request_lens(const TablesLaunch& p, int32_t b) {
  const int32_t most = p.max_pages * kPage;
  Lens r;
  r.seq = min(max(p.seq_lens[b], 0), most);
  r.fresh = min(max(p.new_lens ? p.new_lens[b] : p.q_chunk, 0), r.seq);
  return r;
}
__device__ __forceinline__ int32_t pages_of(int32_t tokens) { return (tokens + kPage - 1) / kPage; }

__global__ __launch_bounds__(kThreads) void step_tables_kernel(TablesLaunch p) {
  __shared__ int32_t row_at[kMaxTableBatch + 1];   // new tokens before request b
  __shared__ int32_t page_at[kMaxTableBatch + 1];  // new pages before request b
  __shared__ int32_t wave_rows[kThreads / 64], wave_pages[kThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;

  // The thread's requests, all their lengths on the way at once.
  const int per = (p.B + kThreads - 1) / kThreads;
  int32_t fresh[kPerThread], need[kPerThread], rows = 0, pages = 0;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    fresh[k] = need[k] = 0;
    if (k < per) {
      const int b = t * per + k;
      const Lens n = request_lens(p, min(b, p.B - 1));
      if (b < p.B) {
        fresh[k] = n.fresh;
        need[k] = pages_of(n.seq) - pages_of(n.seq - n.fresh);
      }
    }
    rows += fresh[k];
    pages += need[k];
  }
  int32_t rows_in = rows, pages_in = pages;  // inclusive over the wave, then the workgroup
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t r = __shfl_up(rows_in, d), g = __shfl_up(pages_in, d);
    if (lane >= d) {
      rows_in += r;
      pages_in += g;
    }
  }
  if (lane == 63) {
    wave_rows[wave] = rows_in;
    wave_pages[wave] = pages_in;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    rows_in += wave_rows[w];
    pages_in += wave_pages[w];
  }
  rows_in -= rows;
  pages_in -= pages;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int b = t * per + k;
    if (k < per && b < p.B) {
      row_at[b] = rows_in;
      page_at[b] = pages_in;
    }
    rows_in += fresh[k];
    pages_in += need[k];
  }
  if (t == kThreads - 1) {
    row_at[p.B] = rows_in;
    page_at[p.B] = pages_in;
  }
  __syncthreads();

  const int32_t total = row_at[p.B];
  const int32_t taken = min(max(p.taken_in[0], 0), p.num_free);
  if (blockIdx.x == 0) {
    for (int b = t; b <= p.B; b += kThreads) p.new_indptr[b] = row_at[b];
    if (t == 0) {
      const int32_t left = p.num_free - taken, need = page_at[p.B];
      p.taken_out[0] = taken + min(need, left);
      p.taken_out[1] = max(need - left, 0);
    }
  }
  const int32_t end = max(total, p.max_tokens);
  for (int64_t row = (int64_t)blockIdx.x * kThreads + t; row < end; row += (int64_t)gridDim.x * kThreads) {
    int32_t slot = -1, pos = 0, request = -1;
    if (row < total) {
      int32_t lo = 0, hi = p.B;  // the last request that starts at or before the row
      while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (row_at[mid] <= row) lo = mid;
        else hi = mid;
      }
      request = lo;
      const Lens n = request_lens(p, lo);
      pos = n.seq - n.fresh + (int32_t)row - row_at[lo];
      const int32_t k = pos / kPage, old = pages_of(n.seq - n.fresh);
      int32_t page;
      if (k >= old) {
        const int32_t left = p.num_free - taken, index = page_at[lo] + k - old;
        page = index < left ? p.free_pages[taken + index] : -1;
        if (pos % kPage == 0) p.block_table[(int64_t)lo * p.max_pages + k] = page;
      } else {
        page = p.block_table[(int64_t)lo * p.max_pages + k];
      }
      if ((uint32_t)page < (uint32_t)p.num_pages) slot = page * kPage + pos % kPage;
    }
    if (row < p.max_tokens) {
      p.slots[row] = slot;
      p.positions[row] = pos;
      p.requests[row] = request;
    }
  }
}

}  // namespace

hipError_t launch_step_tables(const TablesLaunch& p, hipStream_t s) {
  int64_t groups = ((int64_t)p.max_tokens + kRowsPerGroup - 1) / kRowsPerGroup;
  groups = groups < 1 ? 1 : (groups > 256 ? 256 : groups);
  hipLaunchKernelGGL(step_tables_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace splash
