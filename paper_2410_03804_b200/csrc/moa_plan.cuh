// Page tables and slot maps from the requests' lengths (sm_100a): which pages every sequence holds after this step, and where
// each row of the step's packed batch belongs.
//
//   want_b = ceil((len_b + n_b) / page_size), 0 for a sequence that is not in use; pages behind want_b go back to the stack of
//   free pages; who needs more takes them from its top, in the order of the sequences, none overtaking one that waits.
//
// What bounds it: the latency of a chain -- lengths, sums over the sequences, table, rows -- at a decode step's sizes; the stores
// of the maps (16 bytes per row) when whole prompts come in. Two sequences per lane of a warp make the sums; the threads then take
// pages and rows by searching those sums.
// A plan into a second pool overwrites nothing that it reads, so every CTA makes the sums for itself and no two depend on one another:
// one launch over as much of the GPU as there is work for. A page that comes back and is taken at once is read where it was.
// A plan in place has to put pages back before any are taken, and to read before it writes: one CTA, or for large tables a cluster of
// eight, each CTA with its own sums and the cluster's barriers between; the maps of many rows take a second kernel then.
// Measured, calls in a graph, to a second pool: a decode step of 64 sequences 4.1 us (in place 2.9 to 4.3); 64 prompts of up to 32768
// rows (18.4 MB of maps) 7.7 to 8.1 us, where one cluster and a second kernel took 15.1.
#pragma once
#include "moa_paged.cuh"

namespace moa {

constexpr int PL_CLUSTER = 8;
constexpr int PL_THREADS = 512;              // of a plan into a second pool
constexpr int PL_PIECE = 256;

struct PlanArgs {
  const int *table, *held, *free_pages, *free_count;         // [batch, max_pages], [batch], [n_pages] (a stack), [1]
  int *table_out, *held_out, *free_out, *count_out;          // the same ones, or others
  const int *len, *n_new, *seen;                             // [batch]; n_new null: one row each; seen null: len
  int *rows, *row_start, *row_seq, *row_pos;                 // [batch], [batch + 1], [max_rows] twice
  long long* slot;                                           // [max_rows], or null: no maps
  int batch, max_pages, n_pages, shift, max_rows;
  int maps_here;                                             // in place: the first kernel's
  int counts_here;                                           // to a second pool: the first kernel's
};

struct PlanSums {
  int keep[PG_MAX_SEQ], held[PG_MAX_SEQ];
  int take0[PG_MAX_SEQ + 1], back0[PG_MAX_SEQ + 1], row0[PG_MAX_SEQ + 1];         // sums over the sequences before
  int count, have;                                           // free pages before and after those that come back
};

__device__ __forceinline__ int plan_find(const int* start, int x) { return line_seq(start, 1, x); }          // last b with start[b] <= x

template <typename T>
__device__ __forceinline__ T scan_incl(T v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T t = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x & 31) >= o) v += t;
  }
  return v;
}

// One warp. Sums of needs may pass 32 bits; what is granted cannot.
__device__ __forceinline__ void plan_sums(PlanSums& S, const PlanArgs& A) {
  const int lane = threadIdx.x & 31;
  int len[2], n[2], held[2];
  const int count = max(0, min(*A.free_count, A.n_pages));
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int b = lane * 2 + u;
    const bool in = b < A.batch;
    len[u] = in ? A.len[b] : -1;
    n[u] = !in ? 0 : A.n_new ? max(0, A.n_new[b]) : 1;
    held[u] = in ? max(0, min(A.held[b], A.max_pages)) : 0;
  }
  int keep[2], back[2];
  long long need[2];
  bool fits[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const long long want = len[u] < 0 ? 0 : ((long long)len[u] + n[u] + (1 << A.shift) - 1) >> A.shift;
    keep[u] = want < held[u] ? (int)want : held[u];
    back[u] = held[u] - keep[u];
    fits[u] = len[u] >= 0 && want <= A.max_pages;
    need[u] = fits[u] && want > held[u] ? want - held[u] : 0;
  }
  const int back_in = scan_incl(back[0] + back[1]), have = min(count + __shfl_sync(0xffffffffu, back_in, 31), A.n_pages);
  const long long need_in = scan_incl(need[0] + need[1]);
  bool ok[2];
  long long rows[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    ok[u] = fits[u] && (need[u] == 0 || (u ? need_in : need_in - need[1]) <= have);
    rows[u] = ok[u] ? n[u] : 0;
  }
  const long long rows_in = scan_incl(rows[0] + rows[1]);
  int take[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    ok[u] = ok[u] && (u ? rows_in : rows_in - rows[1]) <= A.max_rows;
    take[u] = ok[u] ? (int)need[u] : 0;
    n[u] = ok[u] ? n[u] : 0;
  }
  const int take_in = scan_incl(take[0] + take[1]), row_in = scan_incl(n[0] + n[1]);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int b = lane * 2 + u;
    S.keep[b] = keep[u];
    S.held[b] = held[u];
    S.back0[b] = back_in - back[1] - (u ? 0 : back[0]);
    S.take0[b] = take_in - take[1] - (u ? 0 : take[0]);
    S.row0[b] = row_in - n[1] - (u ? 0 : n[0]);
  }
  if (lane == 31) {
    S.back0[PG_MAX_SEQ] = back_in;
    S.take0[PG_MAX_SEQ] = take_in;
    S.row0[PG_MAX_SEQ] = row_in;
  }
  if (lane == 0) { S.count = count; S.have = have; }
}

// Where row r belongs; page: the entry of a sequence's table.
template <typename Page>
__device__ __forceinline__ void plan_row(const PlanArgs& A, const int* row0, int r, Page page) {
  int b = -1, pos = -1;
  long long at = -1;
  if (r < row0[PG_MAX_SEQ]) {
    b = plan_find(row0, r);
    const int i = r - row0[b], s = A.len[b] + i, p = page(b, s >> A.shift);
    pos = (A.seen ? A.seen[b] : A.len[b]) + i;
    if (p >= 0 && p < A.n_pages) at = ((long long)p << A.shift) + (s & ((1 << A.shift) - 1));
  }
  A.row_seq[r] = b;
  A.row_pos[r] = pos;
  A.slot[r] = at;
}

__device__ __forceinline__ void plan_counts(const PlanSums& S, const PlanArgs& A, int left) {
  const int b = threadIdx.x;
  if (b < A.batch) {
    A.held_out[b] = S.keep[b] + S.take0[b + 1] - S.take0[b];
    A.rows[b] = S.row0[b + 1] - S.row0[b];
  }
  if (b <= A.batch) A.row_start[b] = S.row0[b];
  if (b == 0) *A.count_out = left;
}

// To a second pool.
__global__ void __launch_bounds__(PL_THREADS) page_plan_other_kernel(const PlanArgs A) {
  __shared__ PlanSums S;
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x < 32) plan_sums(S, A);
  __syncthreads();
  const int nt = gridDim.x * blockDim.x, tid = blockIdx.x * blockDim.x + threadIdx.x, left = S.have - S.take0[PG_MAX_SEQ];
  // page i of the stack with the pages that come back on it
  auto stack = [&](int i) {
    if (i < S.count) return A.free_pages[i];
    const int b = plan_find(S.back0, i - S.count);
    return A.table[(size_t)b * A.max_pages + S.keep[b] + (i - S.count - S.back0[b])];
  };
  auto taken = [&](int i) { return stack(S.have - 1 - i); };         // the i-th of all that are taken
  if (A.slot)
#pragma unroll 4
    for (int r = tid; r < A.max_rows; r += nt)
      plan_row(A, S.row0, r, [&](int b, int j) {
        return j < S.keep[b] ? A.table[(size_t)b * A.max_pages + j] : taken(S.take0[b] + j - S.held[b]);
      });
  for (int i = tid; i < S.have; i += nt) A.free_out[i] = stack(i);
  // a warp per PL_PIECE entries of a sequence's table
  const int pieces = (A.max_pages + PL_PIECE - 1) / PL_PIECE;
  for (long long w = tid >> 5; w < (long long)pieces * A.batch; w += nt >> 5) {
    const int b = (int)(w / pieces), j0 = (int)(w - (long long)b * pieces) * PL_PIECE, end = min(j0 + PL_PIECE, A.max_pages);
    const int keep = S.keep[b], held = S.held[b], take0 = S.take0[b], n = S.take0[b + 1] - take0;
    const int* in = A.table + (size_t)b * A.max_pages;
    int* out = A.table_out + (size_t)b * A.max_pages;
#pragma unroll 4
    for (int j = j0 + (tid & 31); j < end; j += 32) out[j] = j < keep ? in[j] : j >= held && j - held < n ? taken(take0 + j - held) : -1;
  }
  if (A.counts_here && blockIdx.x == 0) plan_counts(S, A, left);
}

// Its counts alone, where they overwrite the numbers of new rows that every CTA above makes its sums from.
__global__ void __launch_bounds__(128) page_counts_kernel(const PlanArgs A) {
  __shared__ PlanSums S;
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x < 32) plan_sums(S, A);
  __syncthreads();
  plan_counts(S, A, S.have - S.take0[PG_MAX_SEQ]);
}

// In place.
template <int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(1024) page_plan_kernel(const PlanArgs A) {
  __shared__ PlanSums S;
  pdl_trigger();
  pdl_wait();
  auto barrier = [&]() {
    if constexpr (CL == 1) __syncthreads();
    else asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  const int nt = CL * blockDim.x, tid = blockIdx.x * blockDim.x + threadIdx.x;
  if (threadIdx.x < 32) plan_sums(S, A);
  barrier();                                 // (a CTA's barrier among them) every CTA has read what the next steps overwrite
  const int n_back = S.back0[PG_MAX_SEQ], n_take = S.take0[PG_MAX_SEQ];
  // ---- pages that come back, onto the stack ----
  for (int i = tid; i < n_back; i += nt) {
    const int b = plan_find(S.back0, i), to = S.count + i;
    if (to < A.n_pages) A.free_out[to] = __ldcg(A.table + (size_t)b * A.max_pages + S.keep[b] + (i - S.back0[b]));
  }
  if (CL > 1 || n_back > 0) barrier();
  // ---- pages that are taken, from its top: the i-th of all ----
  auto taken = [&](int i) { return __ldcg((const int*)A.free_out + (S.have - 1 - i)); };
  for (int i = tid; i < n_back; i += nt) {
    const int b = plan_find(S.back0, i);
    A.table_out[(size_t)b * A.max_pages + S.keep[b] + (i - S.back0[b])] = -1;
  }
  for (int i = tid; i < n_take; i += nt) {
    const int b = plan_find(S.take0, i);
    A.table_out[(size_t)b * A.max_pages + S.held[b] + (i - S.take0[b])] = taken(i);
  }
  if (blockIdx.x == 0) plan_counts(S, A, S.have - n_take);
  if (!A.slot || !A.maps_here) return;
  for (int r = tid; r < A.max_rows; r += nt)
    plan_row(A, S.row0, r, [&](int b, int j) {                       // a page that the sequence keeps or one that it takes now
      return j < S.keep[b] ? __ldcg(A.table + (size_t)b * A.max_pages + j) : taken(S.take0[b] + j - S.held[b]);
    });
}

__global__ void __launch_bounds__(256) page_map_kernel(const PlanArgs A) {
  __shared__ int row0[PG_MAX_SEQ + 1];
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x <= PG_MAX_SEQ) row0[threadIdx.x] = A.row_start[min((int)threadIdx.x, A.batch)];
  __syncthreads();
  for (int r = blockIdx.x * blockDim.x + threadIdx.x; r < A.max_rows; r += gridDim.x * blockDim.x)
    plan_row(A, row0, r, [&](int b, int j) { return A.table_out[(size_t)b * A.max_pages + j]; });
}

}  // namespace moa
