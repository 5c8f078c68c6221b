// Eviction from a paged key / value cache by accumulated attention weight (sm_100a).
//
// Per (sequence, head) with L slots in use and a budget m < L, the m slots to keep are: the first positions (pos < sink), the
// latest ones (pos >= seen - recent), and of the others those with the largest weight, a NaN after every number, equal weights
// by the lower slot. A slot on a page that the table does not have holds no row: behind the budget it is given up before all
// others, before the budget it stays where it is and counts, since no row can move there. Keys carry their rotation, so the order of the slots is free: the kept slots behind the budget move into
// the freed slots before it, both in rising order -- at most min(m, L - m) rows move, and no row is both read and written.
//
// What bounds it: the rows that move (4 * dh elements of traffic each), and for small caches the latency of the launch and of
// its dependent steps.
// Few heads: one kernel, a cluster of eight CTAs per (sequence, head), of which every CTA makes the whole selection for
// itself -- reading 8 bytes per slot again costs less than handing the result on -- and moves its share of the rows. The
// cluster's barrier between the two keeps the weights and positions, which may be updated in place, as they were until every
// CTA has read them. Many heads: one CTA per head selects, and a second kernel moves the rows in small shares over the whole
// GPU, since the heads of uneven sequences have uneven numbers of them. Measured, cluster / two kernels, us, heads of 2049 slots cut
// to 2048: 8 heads 8.8 / 9.4, 16: 14.3 / 9.6, 32: 20.9 / 9.8, 64: 33 / 10.0, 128: 59 / 10.2; of 4096 cut to 2048: 8 heads 12.0 / 13.4,
// 16: 21.7 / 15.9, 32: 35 / 20.5, 128: 109 / 37; of 32768 cut to 8192: 8 heads 85 / 91, 16: 165 / 101, 32: 248 / 120. The cluster wins
// while all of them run at once: 14 heads 8.4 / 8.8, 12.0 / 15.1 and (20000 cut to 8192) 55 / 62, but 16 heads a second wave, since
// a group of 16 to 20 SMs holds two clusters only. The rule is ten SMs a head.
// Selection: exact, on 32-bit keys, by up to four passes of 8 bits that end early when a bin is kept whole; then one pass in
// slot order lists sources and destinations.
#pragma once
#include "moa_paged.cuh"

namespace moa {

constexpr int EV_THREADS = 1024;
constexpr int EV_WARPS = EV_THREADS / 32;
constexpr int EV_KEYS = 12288;               // keys kept in shared memory; longer heads read weights and positions again
constexpr int EV_CHUNK = 4 * EV_THREADS;     // slots per step of the ordered pass

struct EvictArgs {
  PagedView c;
  int budget, sink, recent;
  int *n_move, *src, *dst;                   // [batch * hkv], [batch * hkv, list_ld]
  int list_ld;
  float* weight_out;
  int* pos_out;
  int* len_out;                              // or null; not len itself
};

// Rises with the weight; NaN below all numbers, -0 as +0, protected positions above everything. Slots without a page: above
// everything before the budget, lowest of all behind it. So none is a source of a move -- as many slots as the budget have
// higher keys, or all that have a page lie before it -- and none a destination.
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sink, int edge, bool page, bool low) {
  const uint32_t u = __float_as_uint(w + 0.f);
  uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  k = w != w ? 1u : k;
  k = pos < sink || pos >= edge ? 0xffffffffu : k;
  return page ? k : low ? 0xffffffffu : 0u;
}

// Exclusive prefix sum of one value per thread over the CTA; total gets the sum. Ends with a barrier.
__device__ __forceinline__ int evict_scan(int v, int* warp_sum /* EV_WARPS + 1 ints of shared memory */, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    const int own = lane < EV_WARPS ? warp_sum[lane] : 0;
    int s = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += t;
    }
    if (lane < EV_WARPS) warp_sum[lane] = s - own;
    if (lane == 31) warp_sum[EV_WARPS] = s;
  }
  __syncthreads();
  total = warp_sum[EV_WARPS];
  const int r = warp_sum[warp] + inc - v;
  __syncthreads();
  return r;
}

// Moves rows f0 .. f1 - 1 of a head's lists. First a thread per row: its weight and position, and where it comes from and goes
// to (the list, the two pages: dependent loads, made once for all rows side by side), into `at` (WINDOW places of shared
// memory); then the rows, 16 bytes per lane, four steps of a warp under way at a time.
template <typename T, int DH, int NT, int WINDOW>
__device__ __forceinline__ void evict_rows(const EvictArgs& A, int bh, int f0, int f1, longlong2* at) {
  constexpr int CH = DH * (int)sizeof(T) / 16, PER = 32 / CH, UN = 4, E = 16 / (int)sizeof(T), NW = NT / 32;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane % CH, r = lane / CH;
  const int b = bh / A.c.hkv, h = bh - b * A.c.hkv;
  const size_t base = (size_t)bh * (size_t)A.c.cap();
  const int* src = A.src + (size_t)bh * A.list_ld;
  const int* dst = A.dst + (size_t)bh * A.list_ld;
  for (int w0 = f0; w0 < f1; w0 += WINDOW) {
    const int n = min(WINDOW, f1 - w0);
    for (int i = tid; i < n; i += NT) {
      const int s = __ldcg(src + w0 + i), d = __ldcg(dst + w0 + i);
      longlong2 o = make_longlong2(A.c.row(b, s, DH), A.c.row(b, d, DH));      // both are there: see evict_key
      A.weight_out[base + d] = A.c.weight[base + s];
      A.pos_out[base + d] = A.c.pos[base + s];
      o.x = o.y < 0 || o.x < 0 ? -1 : o.x + (long long)h * DH;
      o.y += (long long)h * DH;
      at[i] = o;
    }
    __syncthreads();
    for (int i0 = warp * PER; i0 < n; i0 += UN * NW * PER) {
      uint4 kv[UN], vv[UN];
      long long od[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int i = i0 + r + u * NW * PER;
        const longlong2 o = i < n ? at[i] : make_longlong2(-1, -1);
        od[u] = o.x < 0 ? -1 : o.y + c * E;
        if (o.x >= 0) {
          kv[u] = *reinterpret_cast<const uint4*>((const T*)A.c.k + o.x + c * E);
          vv[u] = *reinterpret_cast<const uint4*>((const T*)A.c.v + o.x + c * E);
        }
      }
#pragma unroll
      for (int u = 0; u < UN; ++u)
        if (od[u] >= 0) {
          *reinterpret_cast<uint4*>((T*)A.c.k + od[u]) = kv[u];
          *reinterpret_cast<uint4*>((T*)A.c.v + od[u]) = vv[u];
        }
    }
    __syncthreads();
  }
}

// CL = 1: selection and lists only.
template <typename T, int DH, int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(EV_THREADS) evict_kernel(const EvictArgs A) {
  pdl_trigger();
  extern __shared__ __align__(16) uint32_t ev_keys[];
  __shared__ int hist[4][256], warp_sum[EV_WARPS + 1];
  __shared__ int s_bin, s_need, s_all;
  const int rank = blockIdx.x % CL, bh = blockIdx.x / CL, b = bh / A.c.hkv, h = bh - b * A.c.hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int cap = (int)A.c.cap(), m = A.budget;
  const int L = min(A.c.len[b], cap);
  const float* wt = A.c.weight + (size_t)bh * cap;
  const int* ps = A.c.pos + (size_t)bh * cap;
  float* wo = A.weight_out + (size_t)bh * cap;
  int* po = A.pos_out + (size_t)bh * cap;
  const bool apart = wo != wt || po != ps;   // outputs of their own: the slots that stay where they are go there too
  if (A.len_out && h == 0 && rank == 0 && tid == 0) A.len_out[b] = min(A.c.len[b], m);
  const bool cut = L > m;
  const int edge = cut ? (int)max(-2147483648ll, (long long)A.c.seen[b] - A.recent) : 0;
  const bool held = L <= EV_KEYS;
  const int* table = A.c.table + (size_t)b * A.c.max_pages;
  auto has_page = [&](int i) { return (unsigned)table[i >> A.c.shift] < (unsigned)A.c.n_pages; };
  auto key_of = [&](int i) { return held ? ev_keys[i] : evict_key(wt[i], ps[i], A.sink, edge, has_page(i), i < m); };
  uint32_t bound = 0u;                       // keys above it are kept, of those equal to it the first `need`
  int shift = 24, need = m, n_equal = 0;
  if (cut) {
    if (held) {
      for (int i = tid; i < L; i += 4 * EV_THREADS) {
        float w[4];
        int p[4];
        bool page[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int j = min(i + u * EV_THREADS, L - 1);
          w[u] = wt[j];
          p[u] = ps[j];
          page[u] = has_page(j);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i + u * EV_THREADS < L) ev_keys[i + u * EV_THREADS] = evict_key(w[u], p[u], A.sink, edge, page[u], i + u * EV_THREADS < m);
      }
    }
    for (int i = tid; i < 4 * 256; i += EV_THREADS) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (;; shift -= 8) {                    // `shift` low bits are still open
      for (int i = tid; i < L; i += EV_THREADS) {
        const uint32_t k = key_of(i);
        if (shift == 24 || ((k ^ bound) >> (shift + 8)) == 0u) atomicAdd(&hist[warp & 3][(k >> shift) & 255u], 1);
      }
      __syncthreads();
      if (warp == 0) {                       // from the top bin down: lane 0 holds bins 255..248, and so on
        int own[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int bin = 255 - (lane * 8 + e);
          own[e] = hist[0][bin] + hist[1][bin] + hist[2][bin] + hist[3][bin];
          sum += own[e];
        }
        int inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += t;
        }
        int above = inc - sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (above < need && above + own[e] >= need) { s_bin = 255 - (lane * 8 + e); s_need = need - above; s_all = own[e]; }
          above += own[e];
        }
      }
      __syncthreads();
      bound |= (uint32_t)s_bin << shift;
      need = s_need;
      n_equal = s_all;
      if (shift == 0 || need == n_equal) break;
      for (int i = tid; i < 4 * 256; i += EV_THREADS) (&hist[0][0])[i] = 0;
      __syncthreads();
    }
  }
  // a key against the bound, on the bits that were decided: 1 above, 0 equal, -1 below
  auto side = [&](uint32_t k) { const uint32_t a = k >> shift, c = bound >> shift; return a > c ? 1 : a == c ? 0 : -1; };
  // ---- every CTA of the head has read weights and positions (its own keys), where they may be written below ----
  const bool ties = need < n_equal;
  int n_move = 0;
  if (cut) {                                 // kept slots behind the budget = freed slots before it
    int eq_base = 0, mine = 0;
    if (!ties) {
      for (int i = tid; i < L - m; i += EV_THREADS) mine += side(key_of(m + i)) >= 0;
    } else {                                 // the slots before the budget decide how many equals are left for those behind it
      int above = 0, equal = 0;
      for (int i = tid; i < m; i += EV_THREADS) equal += side(key_of(i)) == 0;
      for (int i = tid; i < L - m; i += EV_THREADS) above += side(key_of(m + i)) > 0;
      int total;
      (void)evict_scan(equal, warp_sum, total);
      eq_base = max(0, need - total);        // equals kept behind the budget
      mine = above;
    }
    int total;
    (void)evict_scan(mine, warp_sum, total);
    n_move = total + eq_base;
  }
  // this CTA's share of the moves
  const int f0 = (int)((long long)n_move * rank / CL), f1 = (int)((long long)n_move * (rank + 1) / CL);
  int* src = A.src + (size_t)bh * A.list_ld;
  int* dst = A.dst + (size_t)bh * A.list_ld;
  if (cut && n_move > 0) {
    int eq_seen = 0, n_src = 0, n_dst = 0;
    for (int i0 = 0; i0 < L; i0 += EV_CHUNK) {
      const int i = i0 + tid * 4;
      int sd[4], eq = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        sd[u] = i + u < L ? side(key_of(i + u)) : -2;
        eq += sd[u] == 0;
      }
      int total, before = 0;
      if (ties) {
        before = eq_seen + evict_scan(eq, warp_sum, total);
        eq_seen += total;
      }
      unsigned is_src = 0u, is_dst = 0u;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool keep = sd[u] == 1 || (sd[u] == 0 && (!ties || before < need));
        before += sd[u] == 0;
        if (keep && i + u >= m) is_src |= 1u << u;
        if (!keep && sd[u] != -2 && i + u < m) is_dst |= 1u << u;
      }
      // a chunk holds at most 4096 of each: both counts in one scan
      const int at = evict_scan(__popc(is_src) | (__popc(is_dst) << 16), warp_sum, total);
      int s = n_src + (at & 0xffff), d = n_dst + (at >> 16);
      n_src += total & 0xffff;
      n_dst += total >> 16;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if ((is_src >> u) & 1u) { if (s >= f0 && s < f1) src[s] = i + u; ++s; }
        if ((is_dst >> u) & 1u) { if (d >= f0 && d < f1) dst[d] = i + u; ++d; }
      }
    }
  }
  if (apart) {                               // the slots that stay where they are
    const int n = min(L, m);
    for (int i = tid + rank * EV_THREADS; i < n; i += CL * EV_THREADS) {
      // freed slots are written below, by whichever CTA has the move: left out here
      const int sd = cut ? side(key_of(i)) : 1;
      if (sd > 0 || (sd == 0 && !ties)) { wo[i] = wt[i]; po[i] = ps[i]; }
    }
    if (cut && ties) {                       // of the equals the first `need`, counted in slot order
      int eq_seen = 0;
      for (int i0 = 0; i0 < m; i0 += EV_THREADS) {
        const int i = i0 + tid;
        const bool eq = i < m && side(key_of(i)) == 0;
        int total;
        const int before = eq_seen + evict_scan(eq ? 1 : 0, warp_sum, total);
        eq_seen += total;
        if (eq && before < need && rank == 0) { wo[i] = wt[i]; po[i] = ps[i]; }
      }
    }
  }
  if constexpr (CL > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    evict_rows<T, DH, EV_THREADS, EV_KEYS / 4>(A, bh, f0, f1, reinterpret_cast<longlong2*>(ev_keys));     // over the keys
  } else {
    if (tid == 0) A.n_move[bh] = n_move;
  }
}

// The moves of many heads: CTA (share, head).
template <typename T, int DH>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs A, int shares) {
  pdl_trigger();
  __shared__ longlong2 at[512];
  pdl_wait();
  const int bh = blockIdx.x / shares, part = blockIdx.x - bh * shares;
  const long long n = A.n_move[bh];
  evict_rows<T, DH, 256, 512>(A, bh, (int)(n * part / shares), (int)(n * (part + 1) / shares), at);
}

// The new lengths where they replace the old ones: after every head has read those.
__global__ void __launch_bounds__(64) evict_len_kernel(int* len, int batch, int budget) {
  pdl_trigger();
  pdl_wait();
  const int b = threadIdx.x;
  if (b < batch) len[b] = min(len[b], budget);
}

}  // namespace moa
