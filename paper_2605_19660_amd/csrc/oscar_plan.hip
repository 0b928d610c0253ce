// oscar_plan_step: which sequences of a step take part, the pages they give back and get, and where every
// row of the step goes.
//
//   held = ceil(lens / ps), k = min(max(keep, 0), lens), kept = ceil(k / ps)     (ps: tokens of a page)
//   given back : pages kept .. held - 1 of every sequence, in order of sequence and page, on top of the stack
//   fits       : want > 0 and k + want <= ps * max_pages
//   need       = ceil((k + want) / ps) - kept where it fits, else 0
//   takes part : fits, and (need = 0 or the needs up to this sequence are within the stack), and the wants of those
//                up to this sequence are within n_rows
//   pages      : the j-th page handed out, in order of sequence and page, is the j-th from the top
//
// Both sums run over sequences in order and never fall, so that whoever is refused for pages refuses everyone behind
// who needs pages, and whoever is refused for rows everyone behind: the pages handed out are a prefix of the pages
// asked for, and no sequence overtakes one that waits for pages.
//
// What bounds it: a few hundred numbers, so latency.  One workgroup decides (a thread a sequence, sums by scans of
// registers); pages are moved and rows written flat, a thread a page or row, which looks its sequence up in the sums
// in LDS, so that one long prompt costs no more than many tokens.
#include "oscar_common.h"

namespace {

constexpr int MOST_THREADS = 1024;

struct PlanParams {
  const int32_t *lens, *keep, *want;
  int batch, max_pages, num_pages, ps, n_rows;
  int32_t *table, *free_pages;
  const int32_t* n_free;
  int32_t *lens_out, *new_lens, *n_free_out, *row_starts, *positions, *row_seq, *slots;
  int rows_here;   // whether this launch writes the rows
};

// Moved up within a wave, 0 where no lane gives (as permutations through LDS a scan waits for them six times).
template <int CTRL, int ROWS> __device__ __forceinline__ int64_t moved(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// Sum over the threads up to this one, of the workgroup; s_wave: a number a wave that no one else uses meanwhile.
template <int THREADS> __device__ __forceinline__ int64_t group_scan(int64_t v, int64_t* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v += moved<0x111, 0xf>(v);   // row_shr:1, 2, 4, 8
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3
  v += moved<0x143, 0xc>(v);   // row_bcast:31 into rows 2 and 3
  __syncthreads();
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  int64_t before = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) before += w < wave ? s_wave[w] : 0;
  return v + before;
}

// First entry of the non-falling s[0 .. n) that is above x (n if none).
__device__ __forceinline__ int first_above(const int64_t* s, int n, int64_t x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (s[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

struct Seq {
  int64_t len, k, held, kept, want;
};
__device__ __forceinline__ Seq load_seq(const PlanParams& P, int b) {
  Seq s;
  const int64_t most = (int64_t)P.max_pages * P.ps;
  s.len = min(max((int64_t)P.lens[b], (int64_t)0), most);
  s.k = P.keep ? min(max((int64_t)P.keep[b], (int64_t)0), s.len) : s.len;
  s.want = max(P.want[b], 0);
  s.held = (s.len + P.ps - 1) / P.ps;
  s.kept = (s.k + P.ps - 1) / P.ps;
  return s;
}

// One row's entries; b < 0: it belongs to no sequence.
__device__ __forceinline__ void put_row(const PlanParams& P, int64_t row, int b, int pos) {
  if (P.positions) P.positions[row] = b < 0 ? -1 : pos;
  if (P.row_seq) P.row_seq[row] = b;
  if (P.slots) {
    const int page = b < 0 ? -1 : P.table[(int64_t)b * P.max_pages + pos / P.ps];
    P.slots[row] = (uint32_t)page < (uint32_t)P.num_pages ? page * P.ps + pos % P.ps : -1;
  }
}

// THREADS: of the deciding workgroup; a chunk of so many sequences is decided at a time.
template <int THREADS> __global__ __launch_bounds__(THREADS) void oscar_plan_kernel(PlanParams P) {
  __shared__ int64_t s_wave[THREADS / 64], s_sum[THREADS];
  __shared__ int s_kept[THREADS];
  __shared__ int64_t s_most[2];   // rows and pages of the last one that takes part
  const int tid = threadIdx.x;
  const int64_t have = min(max((int64_t)P.n_free[0], (int64_t)0), (int64_t)P.num_pages);
  Seq mine = {};   // of the first chunk
  if (tid < P.batch) mine = load_seq(P, tid);

  // pages that come back
  int64_t avail = have;
  if (P.keep) {
    for (int b0 = 0; b0 < P.batch; b0 += THREADS) {
      const int b = b0 + tid, n = min(P.batch - b0, THREADS);
      Seq s = mine;
      if (b0 > 0) s = tid < n ? load_seq(P, b) : Seq{};
      const int64_t upto = group_scan<THREADS>(s.held - s.kept, s_wave);
      s_sum[tid] = upto;
      s_kept[tid] = (int)s.kept;
      __syncthreads();
      const int64_t total = s_sum[THREADS - 1];
      for (int64_t i = tid; i < total; i += THREADS) {
        const int q = first_above(s_sum, n, i);
        const int64_t col = s_kept[q] + i - (q ? s_sum[q - 1] : 0);
        if (avail + i < P.num_pages) P.free_pages[avail + i] = P.table[(int64_t)(b0 + q) * P.max_pages + col];
      }
      avail = min(avail + total, (int64_t)P.num_pages);
      __syncthreads();
    }
  }

  // who takes part
  int64_t pages_asked = 0, rows_asked = 0, pages_given = 0, rows_given = 0;
  for (int b0 = 0; b0 < P.batch; b0 += THREADS) {
    const int b = b0 + tid, n = min(P.batch - b0, THREADS);
    Seq s = mine;
    if (b0 > 0) s = tid < n ? load_seq(P, b) : Seq{};
    const bool fits = s.want > 0 && s.k + s.want <= (int64_t)P.max_pages * P.ps;
    const int64_t need = fits ? (s.k + s.want + P.ps - 1) / P.ps - s.kept : 0;
    const int64_t pages_upto = pages_asked + group_scan<THREADS>(need, s_wave);
    const bool paged = fits && (need == 0 || pages_upto <= avail);
    const int64_t rows_upto = rows_asked + group_scan<THREADS>(paged ? s.want : 0, s_wave);
    const bool on = paged && rows_upto <= P.n_rows;
    if (tid == 0) s_most[0] = rows_given, s_most[1] = pages_given;
    s_sum[tid] = rows_upto;
    __syncthreads();
    if (on) {   // (the last one's, whoever writes)
      atomicMax(reinterpret_cast<unsigned long long*>(&s_most[0]), (unsigned long long)rows_upto);
      // (one that needs no page may stand behind others that wait for theirs: its sum counts those)
      if (need) atomicMax(reinterpret_cast<unsigned long long*>(&s_most[1]), (unsigned long long)pages_upto);
    }
    const int64_t rows_end = s_sum[THREADS - 1];
    __syncthreads();
    rows_asked = rows_end;
    s_sum[tid] = pages_upto;
    s_kept[tid] = (int)s.kept;
    const int64_t rows_most = s_most[0], pages_most = s_most[1];
    __syncthreads();
    if (tid < n) {
      P.lens_out[b] = (int32_t)(s.k + (on ? s.want : 0));
      P.new_lens[b] = on ? (int32_t)s.want : 0;
      // (behind the last one that takes part both sums have gone past what was given)
      P.row_starts[b] = (int32_t)min(rows_upto - (paged ? s.want : 0), rows_most);
    }
    for (int64_t i = pages_given + tid; i < pages_most; i += THREADS) {
      const int q = first_above(s_sum, n, i);
      const int64_t col = s_kept[q] + i - (q ? s_sum[q - 1] : pages_asked);
      P.table[(int64_t)(b0 + q) * P.max_pages + col] = P.free_pages[avail - 1 - i];
    }
    pages_asked = s_sum[THREADS - 1];
    pages_given = pages_most;
    rows_given = rows_most;
    __syncthreads();
  }
  if (tid == 0) {
    P.row_starts[P.batch] = (int32_t)rows_given;
    P.n_free_out[0] = (int32_t)(avail - pages_given);
  }
  if (!P.rows_here) return;

  // the rows (of one chunk of sequences: oscar_plan_step)
  if (tid < P.batch) {
    s_sum[tid] = P.row_starts[tid] + (int64_t)P.new_lens[tid];   // (this thread's own)
    s_kept[tid] = P.lens_out[tid] - P.new_lens[tid];
  }
  __syncthreads();
  for (int row = tid; row < P.n_rows; row += THREADS) {
    const int q = row < rows_given ? first_above(s_sum, P.batch, row) : -1;
    put_row(P, row, q, q < 0 ? 0 : s_kept[q] + row - (int)(q ? s_sum[q - 1] : 0));
  }
}

__global__ __launch_bounds__(256) void oscar_plan_rows_kernel(PlanParams P) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row >= P.n_rows) return;
  int lo = 0, hi = P.batch;   // first sequence that ends behind the row
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (P.row_starts[mid + 1] > row) hi = mid; else lo = mid + 1;
  }
  if (lo == P.batch)
    put_row(P, row, -1, 0);
  else
    put_row(P, row, lo, P.lens_out[lo] - P.new_lens[lo] + (int)(row - P.row_starts[lo]));
}

}  // namespace

extern "C" int oscar_plan_step(const int32_t* lens, const int32_t* keep, const int32_t* want, int32_t batch,
                               int32_t* block_table, int32_t max_pages_per_seq, int32_t num_pages,
                               int32_t page_size, int32_t* free_pages, const int32_t* n_free, int32_t n_rows,
                               int32_t* lens_out, int32_t* new_lens, int32_t* n_free_out, int32_t* row_starts,
                               int32_t* positions, int32_t* row_seq, int32_t* slots, void* stream) {
  if (batch < 0 || batch > OSCAR_PLAN_MAX_BATCH || max_pages_per_seq < 1 || num_pages < 1 || page_size < 1 || n_rows < 0)
    return OSCAR_ERR_INVALID_ARG;
  // slots and lengths are 32-bit numbers
  if ((int64_t)num_pages * page_size > INT32_MAX || (int64_t)max_pages_per_seq * page_size > INT32_MAX)
    return OSCAR_ERR_INVALID_ARG;
  if (!n_free || !n_free_out || !row_starts || !free_pages) return OSCAR_ERR_INVALID_ARG;
  if (batch > 0 && (!lens || !want || !block_table || !lens_out || !new_lens)) return OSCAR_ERR_INVALID_ARG;
  PlanParams P = {lens, keep, want, batch, max_pages_per_seq, num_pages, page_size, n_rows, block_table, free_pages, n_free,
                  lens_out, new_lens, n_free_out, row_starts, positions, row_seq, slots, 0};
  const bool maps = n_rows > 0 && (positions || row_seq || slots);
  // one workgroup writes some rows a thread beside what else it does; more go to a launch of their own
  const bool small = batch <= 256 && n_rows <= 2048;
  P.rows_here = maps && (small || (n_rows <= 8192 && batch <= MOST_THREADS));
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (small)
    hipLaunchKernelGGL(oscar_plan_kernel<256>, dim3(1), dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL(oscar_plan_kernel<MOST_THREADS>, dim3(1), dim3(MOST_THREADS), 0, st, P);
  if (maps && !P.rows_here)
    hipLaunchKernelGGL(oscar_plan_rows_kernel, dim3((uint32_t)(((int64_t)n_rows + 255) / 256)), dim3(256), 0, st, P);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
