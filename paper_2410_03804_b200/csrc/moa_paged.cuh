// Attention of new rows over a paged key / value cache (sm_100a): one token per sequence, or the rows of a kept draft
// tree, against every cached position and the rows' own uncommitted slots.
//
//   s_j = scale * q . k_j,  p_j = exp(s_j - max s) / sum exp(s - max s),  out = sum_j p_j v_j
//
// Scores, and the running maxima that are taken of them, are kept as the products leave them; only differences from a maximum
// are scaled: exp(scale * (s - max)). So a large scale takes no score out of fp32, and the largest one always gives 1.
//
// What bounds it: one token reads every cached byte once for 4 * group multiply-adds per 4 bytes (bf16), so the cache
// stream from HBM does. The layout follows from that: the queries that share a key / value head -- (rows of the sequence)
// x (heads of the group) -- are stacked 8 to a tile, so a cached row is read once per 8 of them.
//
// Work split (paged_rows_kernel): the (sequence, head, query tile) items are laid end to end as tiles of positions, and
// the CTAs take equal consecutive stretches of that line, whatever the sequences' lengths are; the lengths are read on
// the device, so a captured graph follows them. A stretch may end inside an item: such an item is left in pieces
// (max, sum, unnormalised output), and the CTA that delivers an item's last piece adds them all in the order of their
// positions, the same order on every run. Only the first and the last item of a stretch can be cut, so a CTA has two places
// for pieces: the first for the item its stretch begins in, the second for the one it ends in.
//
// Inside a CTA (one per SM) the eight warps run on their own: each takes every eighth group of positions of the stretch and
// keeps a three-stage ring of its own in shared memory (cp.async, no barrier of the CTA in the loop), with its own running
// maximum, sum and output. The copies run two steps ahead, across the items' borders; at an item's end the warps' states
// are merged through the ring stage that was read last, while the other two fill.
//
// A kernel here may begin while the kernels before it in the stream still write its inputs (programmatic launches), so nothing
// is read through the non-coherent path, whose data may not change while a kernel lives: what is read once comes past L1, the
// rest by ordinary loads.
#pragma once
#include "moa_attn.cuh"

namespace moa {

constexpr int PG_WARPS = 8;
constexpr int PG_THREADS = PG_WARPS * 32;
constexpr int PG_STAGES = 3;
constexpr int PG_ROWS = 8;                   // query rows per tile
constexpr int PG_MAX_SEQ = 64;               // sequences per call

// The cache of one layer as the kernels see it. T [n_pages, page_size, hkv, dh], pages page_stride elements apart.
struct PagedView {
  void *k, *v;
  long long page_stride;
  const int* table;                          // [batch, max_pages]
  const int* len;                            // [batch] committed slots; < 0: the sequence is not in use
  float* weight;                             // [batch, hkv, cap] accumulated weights, or null
  int* pos;                                  // [batch, hkv, cap] position of each slot, or null
  const int* seen;                           // [batch] next position, null when pos is
  int batch, max_pages, n_pages, shift, hkv; // page_size = 1 << shift
  __device__ __forceinline__ long long cap() const { return (long long)max_pages << shift; }
  __device__ __forceinline__ int page_of(int b, long long slot) const { return table[(size_t)b * max_pages + (size_t)(slot >> shift)]; }
  // element offset of (slot, head 0) of sequence b, or -1 where the table has no such page
  __device__ __forceinline__ long long row(int b, long long slot, int dh) const {
    const int page = page_of(b, slot);
    if (page < 0 || page >= n_pages) return -1;
    return page * page_stride + (slot & ((1 << shift) - 1)) * (long long)hkv * dh;
  }
};

struct PagedAttn {
  PagedView c;
  const void* q; long long q_stride;         // row (b, i), head h at q + (b * n + i) * q_stride + h * dh
  const void *k_new, *v_new; long long new_stride;   // the new rows' keys / values, or null: they are in the pages
  const unsigned long long* mask;            // [batch, n] visible new slots of each row, or null: causal
  int n, n_new, hq, group, tiles;            // n_new: visible new slots (0 or n); tiles: query tiles per (sequence, head)
  float scale_log2;
  void* out;                                 // T [batch, n, hq, dh]
  float *part_o, *part_ml;                   // [2 * ctas][rows of an item][dh], the same [2]: pieces
  float* item_ml;                            // [items][PG_ROWS][2]: max and sum of every item, with score
  int* arrived;                              // [ctas]: pieces delivered of the item that is cut first at the end of a CTA's stretch; zero between calls
  float* score; long long score_ld;          // [batch, hq, score_ld] unscaled scores, or null
  int* joins;                                // [ctas][8]: the item that is cut first at the end of a CTA's stretch (tensor-memory kernel)
  float* weight_out;                         // [batch, hkv, cap] or null
  int ctas;                                  // stretches the line is cut into at most
  int min_tiles;                             // ... and the least tiles of one
};

struct PagedLine;
// A place on the line: tile t of item (b, h, mt).
struct PagedPlace {
  int b, h, mt, t, T_b;
  __device__ __forceinline__ void at(const PagedLine& L, const PagedAttn& P, int x);
};

// The line of work: item (b, hm) of sequence b, hm = head * tiles + query tile, has tiles_of(b) tiles of positions and begins
// at pre[b] * hm_n + hm * tiles_of(b). The host keeps the whole line below 2^31 tiles.
struct PagedLine {
  int pre[PG_MAX_SEQ + 1];                   // tiles per item, summed over the sequences before b
  int len[PG_MAX_SEQ];
  int total, ctas, hm_n;                     // tiles of the line, stretches, items per sequence
  // Stretches of equal length wherever they end: the first r of them have q + 1 tiles, the others q. Or, when that costs
  // little, stretches that end where items end: parts[b] of them per item of sequence b, cpre[b] before sequence b.
  int q, r;
  bool whole_items;
  int parts[PG_MAX_SEQ], cpre[PG_MAX_SEQ + 1];
  int x_begin, x_end;                        // this CTA's stretch, empty behind the last, and where it begins
  PagedPlace first;
};

// Every thread of the CTA calls it; ends with a barrier.
__device__ __forceinline__ void paged_line(PagedLine& L, const PagedAttn& P, int tile) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int own[2], sum = 0;
    const int cap = (int)P.c.cap(), hm_n = P.c.hkv * P.tiles;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = lane * 2 + u;
      const int len = b < P.c.batch ? min(P.c.len[b], cap) : -1;
      L.len[b] = len;
      const int keys = len < 0 ? 0 : min(len + P.n_new, cap);
      own[u] = (keys + tile - 1) / tile;
      sum += own[u];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    L.pre[lane * 2] = inc - sum;
    L.pre[lane * 2 + 1] = inc - sum + own[0];
    const int all = __shfl_sync(0xffffffffu, inc, 31), total = all * hm_n;
    const int ctas = max(1, min(P.ctas, (total + P.min_tiles - 1) / P.min_tiles));
    // Whole items: an item's share of the CTAs, rounded down. A stretch that ends inside an item costs its CTA a merge and a
    // new start, about two tiles' time, so they are taken when the longest stretch is at most two tiles longer.
    int n[2], count = 0, worst = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      n[u] = own[u] > 0 ? max(1, (int)((float)ctas * (float)own[u] / (float)total)) : 0;
      count += n[u] * hm_n;
      worst = max(worst, n[u] > 0 ? (own[u] + n[u] - 1) / n[u] : 0);
    }
    worst = __reduce_max_sync(0xffffffffu, worst);
    int cinc = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, cinc, o);
      if (lane >= o) cinc += t;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      L.parts[lane * 2 + u] = n[u];
      L.cpre[lane * 2 + u] = cinc - count + (u ? n[0] * hm_n : 0);
    }
    const int q = total / ctas, r = total - q * ctas;
    const int ccount = __shfl_sync(0xffffffffu, cinc, 31);
    const bool whole_items = ccount <= ctas && worst <= q + 2;
    if (lane == 31) {
      L.pre[PG_MAX_SEQ] = all;
      L.cpre[PG_MAX_SEQ] = ccount;
      L.total = total;
      L.hm_n = hm_n;
      L.q = q;
      L.r = r;
      L.whole_items = whole_items;
      L.ctas = whole_items ? max(1, ccount) : ctas;
    }
    __syncwarp();
    // this CTA's stretch; its sequence is the last one that begins at or before it
    const int cta = blockIdx.x;
    int xb = 0, xe = 0;
    if (total > 0 && cta < L.ctas) {
      const int* pre = whole_items ? L.cpre : L.pre;
      const int scale = whole_items ? 1 : hm_n;
      xb = q * cta + min(cta, r);
      xe = xb + q + (cta < r ? 1 : 0);
      const int key = whole_items ? cta : xb;
      const int b = __popc(__ballot_sync(0xffffffffu, pre[lane] * scale <= key)) + __popc(__ballot_sync(0xffffffffu, pre[lane + 32] * scale <= key)) - 1;
      const int T_b = L.pre[b + 1] - L.pre[b];
      int hm, t;
      if (whole_items) {
        const int np = L.parts[b], k = cta - L.cpre[b], j = k % np, pq = T_b / np, pr = T_b - pq * np;
        hm = k / np;
        t = pq * j + min(j, pr);
        xb = L.pre[b] * hm_n + hm * T_b + t;
        xe = xb + pq + (j < pr ? 1 : 0);
      } else {
        hm = (xb - L.pre[b] * hm_n) / T_b;
        t = xb - L.pre[b] * hm_n - hm * T_b;
      }
      if (lane == 0) {
        L.first.b = b;
        L.first.h = hm / P.tiles;
        L.first.mt = hm - hm / P.tiles * P.tiles;
        L.first.t = t;
        L.first.T_b = T_b;
      }
    }
    if (lane == 0) { L.x_begin = xb; L.x_end = xe; }
  }
  __syncthreads();
}
// the b with pre[b] * scale <= x < pre[b + 1] * scale
__device__ __forceinline__ int line_seq(const int* pre, int scale, int x) {
  int b = 0, hi = PG_MAX_SEQ;
  while (hi - b > 1) {
    const int mid = (b + hi) >> 1;
    if (pre[mid] * scale <= x) b = mid; else hi = mid;
  }
  return b;
}
__device__ __forceinline__ int line_begin(const PagedLine& L, int cta) {
  if (!L.whole_items) return L.q * cta + min(cta, L.r);
  if (cta >= L.ctas) return L.total;
  const int b = line_seq(L.cpre, 1, cta), n = L.parts[b], T_b = L.pre[b + 1] - L.pre[b];
  const int k = cta - L.cpre[b], item = k / n, j = k - item * n, q = T_b / n;
  return L.pre[b] * L.hm_n + item * T_b + q * j + min(j, T_b - q * n);
}
// the CTA whose stretch holds tile x < total
__device__ __forceinline__ int line_owner(const PagedLine& L, int x) {
  int q = L.q, r = L.r, c = 0;
  if (L.whole_items) {
    const int b = line_seq(L.pre, L.hm_n, x), n = L.parts[b], T_b = L.pre[b + 1] - L.pre[b];
    const int in_b = x - L.pre[b] * L.hm_n, item = in_b / T_b;
    x = in_b - item * T_b;
    c = L.cpre[b] + item * n;
    q = T_b / n;
    r = T_b - q * n;
  }
  const int wide = r * (q + 1);
  return c + (x < wide ? x / (q + 1) : r + (x - wide) / q);
}
// The piece that CTA c holds of an item that begins at x0 and that CTA c0 is the first to hold: its first place, unless the
// item begins inside its stretch, which is so for c0 at most. first_place: c0's.
__device__ __forceinline__ int first_place(const PagedLine& L, int c0, int x0) { return line_begin(L, c0) >= x0 ? 0 : 1; }
__device__ __forceinline__ int piece_of(int c, int c0, int first) { return c * 2 + (c == c0 ? first : 0); }

__device__ __forceinline__ void PagedPlace::at(const PagedLine& L, const PagedAttn& P, int x) {
  b = line_seq(L.pre, L.hm_n, x);
  T_b = L.pre[b + 1] - L.pre[b];
  const int in_b = x - L.pre[b] * L.hm_n, hm = in_b / T_b;
  h = hm / P.tiles;
  mt = hm - h * P.tiles;
  t = in_b - hm * T_b;
}

// Which of the new slots some row sees: the others are not read at all (what lies there may be anything).
__device__ __forceinline__ unsigned long long causal_word(int i) { return i >= 63 ? ~0ull : (2ull << i) - 1ull; }
__device__ __forceinline__ unsigned long long any_word(const PagedAttn& P, int b) {          // a whole warp
  if (!P.mask) return causal_word(P.n - 1);
  const int lane = threadIdx.x & 31;
  const unsigned long long* m = P.mask + (size_t)b * P.n;
  unsigned long long a = lane < P.n ? m[lane] : 0ull;
  if (lane + 32 < P.n) a |= m[lane + 32];
  return ((unsigned long long)__reduce_or_sync(0xffffffffu, (unsigned)(a >> 32)) << 32) | __reduce_or_sync(0xffffffffu, (unsigned)a);
}
__device__ __forceinline__ unsigned long long row_word(const PagedAttn& P, int b, int i) {
  return P.mask ? P.mask[(size_t)b * P.n + i] : causal_word(i);
}

// A value that is not finite belongs to the rows that see its slot, and zero times it is not zero. A slot of a tree is seen by
// some rows only: there such values are added to those rows' sums by themselves, and zeros take their place in the products.
__device__ __forceinline__ bool odd_f(float v) { return !(fabsf(v) < INFINITY); }
__device__ __forceinline__ bool odd_lo(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }              // of two bf16 values, the lower one
__device__ __forceinline__ bool odd_hi(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool odd_any(const uint4& x) {
  return odd_lo(x.x) || odd_hi(x.x) || odd_lo(x.y) || odd_hi(x.y) || odd_lo(x.z) || odd_hi(x.z) || odd_lo(x.w) || odd_hi(x.w);
}
__device__ __forceinline__ uint32_t odd_cleared(uint32_t w) { return w & (odd_lo(w) ? 0xffff0000u : ~0u) & (odd_hi(w) ? 0xffffu : ~0u); }
__device__ __forceinline__ uint4 odd_cleared(const uint4& x) { return make_uint4(odd_cleared(x.x), odd_cleared(x.y), odd_cleared(x.z), odd_cleared(x.w)); }

// PagedWarp: one warp's running state over a query tile (maxima of the unscaled scores, sums, outputs, all in fp32), merged over the
// CTA's warps at the end of an item.

// ---------------------------------------------------------------------------------------------
// bf16: mma.sync m16n8k16, 16 positions per warp step, with the positions (then the columns of V) as the 16 rows of the left
// operand and the queries as its 8 columns: S^T = K Q^T, O^T = V^T P^T. A group has 8 query heads at most as a rule, so with
// the queries as the 16 rows half of every product was padding, and the products' issue rate kept 8 warps from getting ahead
// of the cache's stream. Scores and output accumulate in fp32. Probabilities enter the second product as two bf16 terms
// (hi + lo, 16 bits of mantissa): rounding them once to 8 bits would put an error of up to 2^-8 of every term into the output.
// ---------------------------------------------------------------------------------------------
template <typename T, int DH> struct PagedWarp;

// Place of columns d .. d + 7 (d a multiple of 4) of row r in a warp's output of [PG_ROWS][DH] floats.
template <int DH>
__device__ __forceinline__ int pg_at(int r, int d) { return r * DH + ((((d >> 3) ^ r) & (DH / 8 - 1)) << 3) + (d & 7); }

__device__ __forceinline__ uint32_t mat8_trans(uint32_t v) {          // an 8 x 8 matrix of 16-bit values, two per lane, transposed
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <int DH>
struct PagedWarp<bf16, DH> {
  static constexpr int KW = 16;              // positions per warp step
  static constexpr int KS = DH / 16;
  uint32_t qf[KS][2];                        // query gq, columns 16 ks + 2 tq .. and + 8
  float o[DH / 16][4];                       // columns 16 d + gq and + 8 of queries 2 tq and 2 tq + 1
  float m[2], l[2];                          // queries 2 tq, 2 tq + 1; l: this lane's positions
  unsigned long long word[2];                // their mask words
  int gq, tq;

  // The queries' loads may go out while the last item is merged; they are used by the next step.
  static constexpr bool EARLY = true;
  __device__ __forceinline__ void load(const PagedAttn& P, int b, int h, int mt, uint8_t*) {
    const int lane = threadIdx.x & 31;
    gq = lane >> 2; tq = lane & 3;
    const int R = P.n * P.group, r = mt * PG_ROWS + gq;
    const int rc = r < R ? r : 0;            // queries behind the last one are worked on and not written
    const uint32_t* src = reinterpret_cast<const uint32_t*>((const bf16*)P.q + ((long long)b * P.n + rc / P.group) * P.q_stride +
                                                            (long long)(h * P.group + rc % P.group) * DH);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks][0] = src[ks * 8 + tq];
      qf[ks][1] = src[ks * 8 + 4 + tq];
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ bool words(const PagedAttn& P, int b, int mt, int R) {
    bool full = true;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int rr = mt * PG_ROWS + 2 * tq + u;
      word[u] = rr < R ? row_word(P, b, rr / P.group) : 0ull;
      full = full && (rr >= R || word[u] != 0ull);
    }
    return __all_sync(0xffffffffu, full);
  }

  // One step: 16 positions, keys at K, values at V. see(w, j): whether a row with mask word w sees position j of the step;
  // plain: every row sees every position. score: the tile's first row of scores, or null.
  template <bool MANY, typename See>
  __device__ __forceinline__ void step(const PagedAttn& P, const uint8_t* K, uint8_t* V, bool plain, See see, float* score, int, int mt, int R) {
    const int lane = threadIdx.x & 31;
    const uint32_t sK = smem_u32(K), sV = smem_u32(V);
    float s[2][4];                           // two chains halve the products' latency
#pragma unroll
    for (int c = 0; c < 2; ++c) s[c][0] = s[c][1] = s[c][2] = s[c][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint32_t a[4];
      ldsm_x4(sK + tile_off<DH>(lane & 15, ks * 2 + (lane >> 4)), a[0], a[1], a[2], a[3]);
      mma_bf16_16816(s[ks & 1], a, qf[ks][0], qf[ks][1]);
    }
    float z[2][2];                           // [position gq, gq + 8][query 2 tq, 2 tq + 1]
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e >> 1][e & 1] = s[0][e] + s[1][e];
    if (!plain) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!see(word[e & 1], gq + 8 * (e >> 1))) z[e >> 1][e & 1] = -INFINITY;
    }
    if (score) {                             // one token: query = head of the group; for the accumulated weights
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 2 * tq + (e & 1);
        if (mt * PG_ROWS + r < R) score[r * P.score_ld + gq + 8 * (e >> 1)] = z[e >> 1][e & 1];
      }
    }
    float f[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float mx = fmaxf(z[0][u], z[1][u]);
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const float mn = fmaxf(m[u], mx);
      f[u] = (mn == m[u]) ? 1.f : ex2_approx((m[u] - mn) * P.scale_log2);          // m = -inf: 0
      m[u] = mn;
    }
    if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) { o[i][0] *= f[0]; o[i][1] *= f[1]; o[i][2] *= f[0]; o[i][3] *= f[1]; }
      l[0] *= f[0];
      l[1] *= f[1];
    }
    if (MANY && !plain) {
      constexpr int N = KW * DH * 2 / 512;   // 16-byte pieces of the values per lane
      bool odd = false;
#pragma unroll
      for (int u = 0; u < N; ++u) odd = odd || odd_any(reinterpret_cast<const uint4*>(V)[u * 32 + lane]);
      if (__any_sync(0xffffffffu, odd)) {    // (rare)
#pragma unroll 1
        for (int j = 0; j < KW; ++j) {
          const bool s0 = see(word[0], j), s1 = see(word[1], j);
#pragma unroll
          for (int e = 0; e < DH / 8; ++e) {
            const float v = __bfloat162float(*reinterpret_cast<const bf16*>(V + tile_off<DH>(j, e) + gq * 2));
            if (odd_f(v) && s0) o[e >> 1][2 * (e & 1)] += v;
            if (odd_f(v) && s1) o[e >> 1][2 * (e & 1) + 1] += v;
          }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < N; ++u) reinterpret_cast<uint4*>(V)[u * 32 + lane] = odd_cleared(reinterpret_cast<const uint4*>(V)[u * 32 + lane]);
        __syncwarp();
      }
    }
    const float sub0 = m[0] == -INFINITY ? 0.f : m[0], sub1 = m[1] == -INFINITY ? 0.f : m[1];       // seen nothing: exp2(-inf - 0) = 0
    uint32_t hi[2], lo[2];                   // right operand: positions 0..7 and 8..15 x queries
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float p0 = ex2_approx((z[k][0] - sub0) * P.scale_log2), p1 = ex2_approx((z[k][1] - sub1) * P.scale_log2);
      l[0] += p0;
      l[1] += p1;
      const uint32_t w = pack_bf16(p0, p1);
      hi[k] = mat8_trans(w);
      lo[k] = mat8_trans(pack_bf16(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u)));
    }
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
      uint32_t v[4];                         // values transposed: 16 columns x 16 positions
      ldsm_x4_t(sV + tile_off<DH>((lane & 7) + ((lane >> 4) << 3), d * 2 + ((lane >> 3) & 1)), v[0], v[1], v[2], v[3]);
      mma_bf16_16816(o[d], v, hi[0], hi[1]);
      mma_bf16_16816(o[d], v, lo[0], lo[1]);
    }
  }

  // Leaves (max, sum) and the output of the tile's first `rows` queries in shared memory: so [8][DH] (8 columns of a row at the
  // place pg_at gives, so that the rows of a store meet different banks), sml [8][2].
  __device__ __forceinline__ void finish(float* so, float* sml, int rows) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = l[u];
      t += __shfl_xor_sync(0xffffffffu, t, 4);
      t += __shfl_xor_sync(0xffffffffu, t, 8);
      t += __shfl_xor_sync(0xffffffffu, t, 16);
      const int r = 2 * tq + u;
      if (r >= rows) continue;
      if (gq == 0) { sml[r * 2] = m[u]; sml[r * 2 + 1] = t; }
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) {
        so[pg_at<DH>(r, i * 16) + gq] = o[i][u];
        so[pg_at<DH>(r, i * 16 + 8) + gq] = o[i][2 + u];
      }
    }
  }
};

// ---------------------------------------------------------------------------------------------
// fp32: plain multiply-adds, 8 positions per warp step. Scores: a lane takes one position and a quarter of the columns
// (chunks quarter, quarter + 4, ... so that the four quarters read different banks); outputs: a lane takes DH / 32
// neighbouring columns of all rows.
// ---------------------------------------------------------------------------------------------
template <int DH>
struct PagedWarp<float, DH> {
  static constexpr int KW = 8;
  static constexpr int DL = DH / 32;         // output columns per lane
  float o[PG_ROWS][DL];
  float *sq, *sp;                            // queries of the CTA, this warp's probabilities
  int rows;                                  // query rows of this tile

  // Shared memory behind the rings: queries of the item [PG_ROWS][DH], then per warp probabilities [KW][PG_ROWS] and factors.
  static constexpr int SMEM = (PG_ROWS * DH + PG_WARPS * (KW + 1) * PG_ROWS) * 4;

  float mrow, lrow;                          // running max and sum of row lane % PG_ROWS; the lanes of a row hold the same

  static constexpr bool EARLY = false;       // the queries are shared by the warps
  __device__ __forceinline__ void load(const PagedAttn& P, int b, int h, int mt, uint8_t* extra) {
    const int R = P.n * P.group;
    sq = reinterpret_cast<float*>(extra);
    sp = sq + PG_ROWS * DH + (threadIdx.x >> 5) * (KW + 1) * PG_ROWS;
    rows = min(PG_ROWS, R - mt * PG_ROWS);
    for (int i = threadIdx.x; i < PG_ROWS * DH / 4; i += PG_THREADS) {
      const int rl = i / (DH / 4), c = i - rl * (DH / 4);
      const int r = mt * PG_ROWS + rl;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < R)
        x = reinterpret_cast<const float4*>((const float*)P.q + ((long long)b * P.n + r / P.group) * P.q_stride + (long long)(h * P.group + r % P.group) * DH)[c];
      reinterpret_cast<float4*>(sq)[i] = x;
    }
    __syncthreads();
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r)
#pragma unroll
      for (int d = 0; d < DL; ++d) o[r][d] = 0.f;
    mrow = -INFINITY;
    lrow = 0.f;
  }

  // 16-byte chunk of a row, swizzled by the row
  static __device__ __forceinline__ uint32_t off(int row, int chunk) { return (uint32_t)(row * (DH * 4) + ((chunk ^ (row & 7)) << 4)); }

  __device__ __forceinline__ bool words(const PagedAttn& P, int b, int mt, int R) {
    const int rr = mt * PG_ROWS + (threadIdx.x & (PG_ROWS - 1));
    return __all_sync(0xffffffffu, rr >= R || row_word(P, b, rr / P.group) != 0ull);
  }

  template <bool MANY, typename See>
  __device__ __forceinline__ void step(const PagedAttn& P, const uint8_t* K, uint8_t* V, bool plain, See see, float* score, int b, int mt, int) {
    const int lane = threadIdx.x & 31;
    const int kk = lane & 7, quarter = lane >> 3;
    float acc[PG_ROWS];
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r) acc[r] = 0.f;
#pragma unroll 2
    for (int c = quarter; c < DH / 4; c += 4) {
      const float4 x = *reinterpret_cast<const float4*>(K + off(kk, c));
#pragma unroll
      for (int r = 0; r < PG_ROWS; ++r) {
        if (r >= rows) break;
        const float4 y = *reinterpret_cast<const float4*>(sq + r * DH + c * 4);
        acc[r] = fmaf(x.x, y.x, acc[r]);
        acc[r] = fmaf(x.y, y.y, acc[r]);
        acc[r] = fmaf(x.z, y.z, acc[r]);
        acc[r] = fmaf(x.w, y.w, acc[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r) {
      if (r >= rows) break;
      float t = acc[r];
      t += __shfl_xor_sync(0xffffffffu, t, 8);
      t += __shfl_xor_sync(0xffffffffu, t, 16);
      if (quarter == (r & 3)) sp[kk * PG_ROWS + r] = (plain || see(row_word(P, b, (mt * PG_ROWS + r) / P.group), kk)) ? t : -INFINITY;
    }
    __syncwarp();
    // softmax statistics: lane r holds row r % PG_ROWS
    {
      const int r = lane & (PG_ROWS - 1);
      float z[KW], mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        z[k] = r < rows ? sp[k * PG_ROWS + r] : -INFINITY;
        mx = fmaxf(mx, z[k]);
      }
      if (score && lane < PG_ROWS && r < rows) {
#pragma unroll
        for (int k = 0; k < KW; k += 4) *reinterpret_cast<float4*>(score + r * P.score_ld + k) = make_float4(z[k], z[k + 1], z[k + 2], z[k + 3]);
      }
      const float mn = fmaxf(mrow, mx);
      const float f = mn == mrow ? 1.f : exp2f((mrow - mn) * P.scale_log2);
      mrow = mn;
      const float sub = mn == -INFINITY ? 0.f : mn;
      lrow *= f;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float p = exp2f((z[k] - sub) * P.scale_log2);
        lrow += p;
        if (lane < PG_ROWS) sp[k * PG_ROWS + r] = p;
      }
      if (lane < PG_ROWS) sp[KW * PG_ROWS + r] = f;
      if (__any_sync(0xffffffffu, f != 1.f)) {
        __syncwarp();
#pragma unroll
        for (int q = 0; q < PG_ROWS; ++q) {
          const float g = sp[KW * PG_ROWS + q];
#pragma unroll
          for (int d = 0; d < DL; ++d) o[q][d] *= g;
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      float v[DL];
      if constexpr (DL == 4) {
        const float4 t = *reinterpret_cast<const float4*>(V + off(k, lane));
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
      } else {
        const float2 t = *reinterpret_cast<const float2*>(V + off(k, lane >> 1) + (lane & 1) * 8);
        v[0] = t.x; v[1] = t.y;
      }
      if (MANY && !plain) {
#pragma unroll
        for (int d = 0; d < DL; ++d)
          if (odd_f(v[d])) {                 // (rare)
#pragma unroll
            for (int r = 0; r < PG_ROWS; ++r)
              if (r < rows && see(row_word(P, b, (mt * PG_ROWS + r) / P.group), k)) o[r][d] += v[d];
            v[d] = 0.f;
          }
      }
#pragma unroll
      for (int r = 0; r < PG_ROWS; r += 4) {
        if (r >= rows) break;
        const float4 p = *reinterpret_cast<const float4*>(sp + k * PG_ROWS + r);
#pragma unroll
        for (int d = 0; d < DL; ++d) {
          o[r][d] = fmaf(p.x, v[d], o[r][d]);
          o[r + 1][d] = fmaf(p.y, v[d], o[r + 1][d]);
          o[r + 2][d] = fmaf(p.z, v[d], o[r + 2][d]);
          o[r + 3][d] = fmaf(p.w, v[d], o[r + 3][d]);
        }
      }
    }
    __syncwarp();
  }

  __device__ __forceinline__ void finish(float* so, float* sml, int) {
    const int lane = threadIdx.x & 31;
    if (lane < PG_ROWS) { sml[lane * 2] = mrow; sml[lane * 2 + 1] = lrow; }
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r)
#pragma unroll
      for (int d = 0; d < DL; ++d) so[pg_at<DH>(r, lane * DL) + d] = o[r][d];
  }
};

template <typename T, int DH> struct PagedCfg {
  static constexpr int KW = PagedWarp<T, DH>::KW;
  static constexpr int TILE = PG_WARPS * KW;                    // positions per CTA step
  static constexpr int E = 16 / (int)sizeof(T);                 // elements per 16 bytes
  static constexpr int CH = DH / E;                             // 16-byte chunks per row
  static constexpr int ROW_BYTES = DH * (int)sizeof(T);
  static constexpr int HALF = KW * ROW_BYTES;                   // a warp's keys (or values) of one stage
  static constexpr int STAGE = 2 * HALF;
  static constexpr int RING = PG_STAGES * STAGE;                // of one warp
  static constexpr int EXTRA = sizeof(T) == 4 ? PagedWarp<float, DH>::SMEM : 0;
  static constexpr int SMEM = PG_WARPS * RING + EXTRA;
  static_assert(PG_ROWS * DH * 4 <= STAGE, "a warp's output takes the place of one stage of its ring");
};

template <typename T>
__device__ __forceinline__ void store4(T* dst, const float4 a) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
  else *reinterpret_cast<float4*>(dst) = a;
}

// MANY: more than one row per sequence, so that some rows may see a slot that others do not (those steps inline cost a token's
// call 2 %).
template <typename T, int DH, bool MANY>
__global__ void __launch_bounds__(PG_THREADS, 1) paged_rows_kernel(const PagedAttn P) {
  using C = PagedCfg<T, DH>;
  pdl_trigger();
  extern __shared__ __align__(128) uint8_t pg_smem[];
  __shared__ PagedLine L;
  __shared__ unsigned int live_of[PG_WARPS][PG_STAGES];
  __shared__ float sml[PG_WARPS][PG_ROWS][2];
  __shared__ int s_last[2], s_join[2][6];    // cut items of this CTA: whether it delivered the last piece; x0, b, h, mt, first and last CTA
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const extra = pg_smem + PG_WARPS * C::RING;
  uint8_t* const ring = pg_smem + warp * C::RING;
  const uint32_t ring_s = smem_u32(ring);
  pdl_wait(KID_ATTN);
  paged_line(L, P, C::TILE);
  const int x_begin = L.x_begin, x_end = L.x_end;
  if (x_begin == x_end) return;
  if (threadIdx.x < 2) s_last[threadIdx.x] = 0;
  const int R = P.n * P.group;
  const int cap = (int)P.c.cap();

  // ---- copies: place of the next step that is asked for, two steps ahead of the one that is worked on ----
  PagedPlace F = L.first;
  int f_x = x_begin, f_len = L.len[F.b], f_keys = min(f_len + P.n_new, cap);
  unsigned long long f_any = any_word(P, F.b);
  const int ch = lane % C::CH, r_first = lane / C::CH;
  constexpr int R_STEP = 32 / C::CH;
  // A step's rows -> this warp's ring. A row that does not exist is zero-filled: zero times what lies there may not be zero.
  // look() finds the row of this lane's position of step F and moves F on; a step ahead of the copies that use it, so that they
  // do not wait for the table.
  long long off = 0;
  int src = 0;                                // src 0: does not exist, 1: page, 2: new row
  auto look = [&]() {
    src = 0;
    if (f_x >= x_end) return;
    const int key = F.t * C::TILE + warp * C::KW + lane;
    if (lane < C::KW && key < f_keys) {
      if (key >= f_len && !((f_any >> (key - f_len)) & 1ull)) {
        src = 0;
      } else {
        off = P.c.row(F.b, key, DH);
        src = off >= 0 ? 1 : 0;
        off += (long long)F.h * DH;
        if (src != 0 && key >= f_len && P.k_new) {                   // a new row whose page the table does not have is left out, too
          src = 2;
          off = ((long long)F.b * P.n + (key - f_len)) * P.new_stride + (long long)F.h * DH;
        }
      }
    }
    if (++F.t == F.T_b && f_x + 1 < x_end) {
      F.at(L, P, f_x + 1);
      f_len = L.len[F.b];
      f_keys = min(f_len + P.n_new, cap);
      f_any = any_word(P, F.b);
    }
  };
  auto issue = [&](int st) {
    const uint32_t dK = ring_s + st * C::STAGE, dV = dK + C::HALF;
    const unsigned live = __ballot_sync(0xffffffffu, src != 0), fresh = __ballot_sync(0xffffffffu, src == 2);
    if (lane == 0) live_of[warp][st] = live;
#pragma unroll
    for (int r0 = 0; r0 < C::KW; r0 += R_STEP) {
      const int r = r0 + r_first;
      const long long o = __shfl_sync(0xffffffffu, off, r);
      const bool ok = (live >> r) & 1u, nw = (fresh >> r) & 1u;
      const T* kp = (const T*)(nw ? P.k_new : P.c.k) + (ok ? o : 0) + ch * C::E;
      const T* vp = (const T*)(nw ? P.v_new : P.c.v) + (ok ? o : 0) + ch * C::E;
      const uint32_t d = (uint32_t)(r * C::ROW_BYTES + ((ch ^ (r & 7)) << 4));
      cp_async16(dK + d, kp, ok);
      cp_async16(dV + d, vp, ok);
    }
    ++f_x;
    look();
  };
  look();
  PagedWarp<T, DH> W;
  PagedPlace S = L.first;
  W.load(P, S.b, S.h, S.mt, extra);                                  // the first queries are on their way before the copies
#pragma unroll
  for (int st = 0; st < PG_STAGES - 1; ++st) {
    if (f_x < x_end) issue(st);
    cp_async_commit();
  }
  int st = 0;
  for (int x = x_begin; x < x_end;) {
    if (x != x_begin) S.at(L, P, x);
    const int b = S.b, h = S.h, mt = S.mt, t0 = S.t, t1 = min(S.T_b, t0 + (x_end - x));
    const int x0 = x - t0;                                           // the item's first tile on the line
    const int len = L.len[b], keys = min(len + P.n_new, cap);
    if (x != x_begin && !W.EARLY) W.load(P, b, h, mt, extra);
    W.clear();
    const bool full_rows = W.words(P, b, mt, R);                     // every row of this warp's tile sees the committed slots
    const bool whole = t0 == 0 && t1 == S.T_b;
    const int place = x == x_begin ? 0 : 1;
    if (!whole && threadIdx.x == PG_THREADS - 32) {                  // (while the first copies are on their way)
      int* j = s_join[place];
      j[0] = x0; j[1] = b; j[2] = h; j[3] = mt;
      j[4] = place ? (int)blockIdx.x : line_owner(L, x0);
      j[5] = line_owner(L, x0 + S.T_b - 1);
    }
    for (int t = t0; t < t1; ++t) {
      if (f_x < x_end) issue(st == 0 ? PG_STAGES - 1 : st - 1);      // the stage of the step before this one
      cp_async_commit();
      cp_async_wait<PG_STAGES - 1>();
      __syncwarp();
      const int base = t * C::TILE + warp * C::KW;
      const unsigned live = live_of[warp][st];
      if (live != 0u) {
        uint8_t* sK = ring + st * C::STAGE;
        uint8_t* sV = sK + C::HALF;
        constexpr unsigned ALL = (1u << C::KW) - 1u;
        const bool plain = live == ALL && base + C::KW <= len && full_rows;
        // whether a row with mask word w sees position base + j
        auto sees = [&](unsigned long long w, int j) -> bool {
          if (!((live >> j) & 1u)) return false;
          const int key = base + j;
          return key < len ? w != 0ull : ((w >> (key - len)) & 1ull) != 0ull;
        };
        // the item's first query tile writes the new rows it holds to their pages
        if (P.k_new && mt == 0 && base + C::KW > len) {
          for (int r = r_first; r < C::KW; r += R_STEP) {
            const int key = base + r;
            if (key < len || key >= keys || !((live >> r) & 1u)) continue;
            const long long o = P.c.row(b, key, DH);
            if (o < 0) continue;
            const uint32_t d = (uint32_t)(r * C::ROW_BYTES + ((ch ^ (r & 7)) << 4));
            *reinterpret_cast<uint4*>((T*)P.c.k + o + (long long)h * DH + ch * C::E) = *reinterpret_cast<const uint4*>(sK + d);
            *reinterpret_cast<uint4*>((T*)P.c.v + o + (long long)h * DH + ch * C::E) = *reinterpret_cast<const uint4*>(sV + d);
          }
        }
        float* at = P.score ? P.score + ((long long)b * P.hq + h * P.group + mt * PG_ROWS) * P.score_ld + base : nullptr;
        W.template step<MANY>(P, sK, sV, plain, sees, at, b, mt, R);
      } else if (P.score && base < keys) {                           // nothing there: the weights' pass reads -inf
        for (int i = lane; i < C::KW * min(PG_ROWS, R - mt * PG_ROWS); i += 32)
          P.score[((long long)b * P.hq + h * P.group + mt * PG_ROWS + i / C::KW) * P.score_ld + base + i % C::KW] = -INFINITY;
      }
      if (P.k_new && mt == 0 && P.c.pos && base + C::KW > len && lane < C::KW) {
        const int key = base + lane;
        if (key >= len && key < keys) {
          const size_t at = ((size_t)b * P.c.hkv + h) * (size_t)cap + (size_t)key;
          P.c.pos[at] = P.c.seen[b] + (key - len);
          P.c.weight[at] = 0.f;
        }
      }
      __syncwarp();
      if (t + 1 < t1) st = st == PG_STAGES - 1 ? 0 : st + 1;
    }
    // ---- merge of the warps, through the stage that was read last; the next item's queries set out before ----
    const int rows = min(PG_ROWS, R - mt * PG_ROWS), xn = x + (t1 - t0);
    if (W.EARLY && xn < x_end) {
      PagedPlace N = S;
      N.at(L, P, xn);
      W.load(P, N.b, N.h, N.mt, extra);
    }
    W.finish(reinterpret_cast<float*>(ring + st * C::STAGE), &sml[warp][0][0], rows);
    __syncthreads();
    const int item = (b * P.c.hkv + h) * P.tiles + mt;
    const size_t prow = ((size_t)blockIdx.x * 2 + place) * PG_ROWS;
    for (int i = threadIdx.x; i < rows * (DH / 4); i += PG_THREADS) {
      const int r = i / (DH / 4), c = i - r * (DH / 4), rr = mt * PG_ROWS + r;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < PG_WARPS; ++w) M = fmaxf(M, sml[w][r][0]);
      const float ref = M == -INFINITY ? 0.f : M;
      float Z = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < PG_WARPS; ++w) {
        const float f = exp2f((sml[w][r][0] - ref) * P.scale_log2);
        Z = fmaf(f, sml[w][r][1], Z);
        const float4 y = *reinterpret_cast<const float4*>(pg_smem + w * C::RING + st * C::STAGE + pg_at<DH>(r, c * 4) * 4);
        a.x = fmaf(f, y.x, a.x); a.y = fmaf(f, y.y, a.y); a.z = fmaf(f, y.z, a.z); a.w = fmaf(f, y.w, a.w);
      }
      if (whole) {
        const float inv = Z == 0.f ? 0.f : 1.f / Z;                  // a row that sees nothing; a NaN stays one
        if (Z == 0.f) a = make_float4(0.f, 0.f, 0.f, 0.f);
        store4((T*)P.out + (((size_t)b * P.n + rr / P.group) * P.hq + h * P.group + rr % P.group) * DH + c * 4,
               make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
        if (c == 0 && P.score) { P.item_ml[((size_t)item * PG_ROWS + r) * 2] = M; P.item_ml[((size_t)item * PG_ROWS + r) * 2 + 1] = Z; }
      } else {
        __stcg(reinterpret_cast<float4*>(P.part_o + (prow + r) * DH + c * 4), a);
        if (c == 0) __stcg(reinterpret_cast<float2*>(P.part_ml + (prow + r) * 2), make_float2(M, Z));
      }
    }
    __syncthreads();                                                 // the merge is read before its stage fills again
    if (!whole && threadIdx.x == 0) {
      // The piece is delivered; who delivers an item's last one joins them, at the end, when nothing else waits for it. (The
      // barrier and this thread's fence order the CTA's stores before the count.)
      const int c0 = s_join[place][4], c1 = s_join[place][5];
      __threadfence();
      s_last[place] = atomicAdd(P.arrived + c0, 1) == c1 - c0;
    }
    x = xn;
    st = st == PG_STAGES - 1 ? 0 : st + 1;
  }

  // ---- join: pieces in the order of their positions, a group of threads for every so many of them ----
  __syncthreads();
  for (int place = 0; place < 2; ++place) {
    if (!s_last[place]) continue;                                    // the same for the whole CTA
    const int x0 = s_join[place][0], b = s_join[place][1], h = s_join[place][2], mt = s_join[place][3], c0 = s_join[place][4], c1 = s_join[place][5];
    if (threadIdx.x == 0) P.arrived[c0] = 0;                         // as the next call expects it
    __threadfence();
    const int rows = min(PG_ROWS, R - mt * PG_ROWS), units = rows * (DH / 4), np = c1 - c0 + 1;
    const int fp = first_place(L, c0, x0);
    const int subs = max(1, min(PG_THREADS / units, (np + 7) / 8)), each = (np + subs - 1) / subs;
    float* sub_o = reinterpret_cast<float*>(pg_smem);                // [sub][unit][6]; the rings are empty
    for (int u0 = 0; u0 < units; u0 += PG_THREADS) {
      const int sub = threadIdx.x / units, unit = subs > 1 ? threadIdx.x - sub * units : u0 + threadIdx.x;
      const bool work = sub < subs && unit < units;
      const int r = unit / (DH / 4), c = unit - r * (DH / 4), rr = mt * PG_ROWS + r;
      float M = -INFINITY, Z = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      auto add = [&](float m, float z, const float4& o, float ref) {
        const float f = exp2f((m - ref) * P.scale_log2);
        Z = fmaf(f, z, Z);
        a.x = fmaf(f, o.x, a.x); a.y = fmaf(f, o.y, a.y); a.z = fmaf(f, o.z, a.z); a.w = fmaf(f, o.w, a.w);
      };
      if (work) {
        const int p_end = min(c1 + 1, c0 + (sub + 1) * each);
        for (int p0 = c0 + sub * each; p0 < p_end; p0 += 8) {        // eight loads under way; the sums move to a new reference
          float2 ml[8];
          float4 o[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const size_t at = (size_t)piece_of(min(p0 + u, p_end - 1), c0, fp) * PG_ROWS + r;
            ml[u] = __ldcg(reinterpret_cast<const float2*>(P.part_ml + at * 2));
            o[u] = __ldcg(reinterpret_cast<const float4*>(P.part_o + at * DH + c * 4));
          }
          float mx = M;
#pragma unroll
          for (int u = 0; u < 8; ++u) mx = fmaxf(mx, ml[u].x);
          const float ref = mx == -INFINITY ? 0.f : mx, g = exp2f((M - ref) * P.scale_log2);
          Z *= g;
          a.x *= g; a.y *= g; a.z *= g; a.w *= g;
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (p0 + u < p_end) add(ml[u].x, ml[u].y, o[u], ref);
          M = mx;
        }
      }
      if (subs > 1) {                                                // units <= the CTA's threads: one round
        float* t = sub_o + (sub * units + unit) * 6;
        if (work && sub > 0) { t[0] = M; t[1] = Z; t[2] = a.x; t[3] = a.y; t[4] = a.z; t[5] = a.w; }
        __syncthreads();
        if (work && sub == 0) {
          float mx = M;
          for (int q = 1; q < subs; ++q) mx = fmaxf(mx, sub_o[(q * units + unit) * 6]);
          const float ref = mx == -INFINITY ? 0.f : mx, g = exp2f((M - ref) * P.scale_log2);
          Z *= g;
          a.x *= g; a.y *= g; a.z *= g; a.w *= g;
          for (int q = 1; q < subs; ++q) {
            const float* y = sub_o + (q * units + unit) * 6;
            add(y[0], y[1], make_float4(y[2], y[3], y[4], y[5]), ref);
          }
          M = mx;
        }
        __syncthreads();
      }
      if (work && sub == 0) {
        const float inv = Z == 0.f ? 0.f : 1.f / Z;
        if (Z == 0.f) a = make_float4(0.f, 0.f, 0.f, 0.f);
        store4((T*)P.out + (((size_t)b * P.n + rr / P.group) * P.hq + h * P.group + rr % P.group) * DH + c * 4,
               make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
        const int item = (b * P.c.hkv + h) * P.tiles + mt;
        if (c == 0 && P.score) { P.item_ml[((size_t)item * PG_ROWS + r) * 2] = M; P.item_ml[((size_t)item * PG_ROWS + r) * 2 + 1] = Z; }
      }
    }
  }
}

// Rows of sequences in use that have no position at all: zeros. One CTA per sequence, only where that can happen.
template <typename T>
__global__ void __launch_bounds__(256) paged_empty_kernel(T* out, const int* len, int batch, int per_seq) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x;
  if (len[b] != 0) return;
  for (int d = threadIdx.x; d < per_seq; d += 256) out[(size_t)b * per_seq + d] = from_f<T>(0.f);
}

// weight_out = weight + sum over the group's heads of exp(scale * (score - max)) / sum, for those of slots 0 .. keys - 1 of every
// (sequence, head) that the row sees, 256 slots per CTA at a time; a thread's scores of eight heads are under way together.
__global__ void __launch_bounds__(256) paged_weights_kernel(const PagedAttn P) {
  pdl_trigger();
  constexpr int CHUNK = 256;
  __shared__ int pre[PG_MAX_SEQ + 1], s_len[PG_MAX_SEQ];
  __shared__ float2 ml[128];                 // per head: maximum, 1 / sum
  pdl_wait();
  const int cap = (int)P.c.cap();
  if (threadIdx.x < 32) {                    // chunks per head, summed over the sequences before
    const int lane = threadIdx.x;
    int own[2], sum = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = lane * 2 + u, len = b < P.c.batch ? min(P.c.len[b], cap) : -1;
      s_len[b] = len;
      own[u] = len < 0 ? 0 : (min(len + P.n_new, cap) + CHUNK - 1) / CHUNK;
      sum += own[u];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    pre[lane * 2] = inc - sum;
    pre[lane * 2 + 1] = inc - sum + own[0];
    if (lane == 31) pre[PG_MAX_SEQ] = inc;
  }
  __syncthreads();
  const int n_chunks = pre[PG_MAX_SEQ] * P.c.hkv;
  for (int w = blockIdx.x; w < n_chunks; w += gridDim.x) {
    const int b = line_seq(pre, P.c.hkv, w), per = pre[b + 1] - pre[b], in_b = w - pre[b] * P.c.hkv, h = in_b / per;
    const int slot = (in_b - h * per) * CHUNK + threadIdx.x, keys = min(s_len[b] + P.n_new, cap);
    const size_t at = ((size_t)b * P.c.hkv + h) * (size_t)cap + slot;
    const float* score = P.score + ((long long)b * P.hq + h * P.group) * P.score_ld + slot;
    const bool in = slot < keys;
    const int page = in ? P.c.page_of(b, slot) : -1;
    const unsigned long long word = row_word(P, b, 0);               // one row; bit 0: its own slot
    const float old = in && P.c.weight && slot < s_len[b] ? P.c.weight[at] : 0.f;
    float z[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) z[u] = in && u < P.group ? __ldcg(score + u * P.score_ld) : -INFINITY;
    if (threadIdx.x < P.group) {
      const float2 t = __ldcg(reinterpret_cast<const float2*>(P.item_ml) + (size_t)(b * P.c.hkv + h) * P.tiles * PG_ROWS + threadIdx.x);
      ml[threadIdx.x] = make_float2(t.x == -INFINITY ? 0.f : t.x, t.y == 0.f ? 0.f : 1.f / t.y);
    }
    __syncthreads();
    float sum = 0.f;
    for (int g0 = 0; g0 < P.group; g0 += 8) {
      if (g0 > 0) {
#pragma unroll
        for (int u = 0; u < 8; ++u) z[u] = in && g0 + u < P.group ? __ldcg(score + (g0 + u) * P.score_ld) : -INFINITY;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (g0 + u < P.group) sum = fmaf(exp2f((z[u] - ml[g0 + u].x) * P.scale_log2), ml[g0 + u].y, sum);
    }
    if (page >= 0 && page < P.c.n_pages && (slot < s_len[b] ? word != 0ull : (word & 1ull) != 0ull)) P.weight_out[at] = old + sum;
    __syncthreads();
  }
}

// Writes rows i < n_new[b] of k_new / v_new [batch, n, hkv, dh] (row_stride elements apart) to slots len[b] + i; with mask
// [batch, n] only those that some row sees. 16 bytes per thread.
template <typename T>
__global__ void __launch_bounds__(256) paged_append_kernel(PagedView C, const T* k_new, const T* v_new, long long row_stride, int n,
                                                           const int* n_new, const unsigned long long* mask, int dh) {
  pdl_trigger();
  pdl_wait(KID_APPEND);
  constexpr int E = 16 / sizeof(T);
  const int b = blockIdx.y, per = C.hkv * dh / E;
  const int len = C.len[b];
  if (len < 0) return;
  const int rows = n_new ? min(n, n_new[b]) : n;
  unsigned long long any = ~0ull;
  if (mask) {                                                        // n <= 64
    any = 0ull;
    for (int i = 0; i < n; ++i) any |= mask[(size_t)b * n + i];
  }
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)rows * per; i += (long long)gridDim.x * blockDim.x) {
    const int r = (int)(i / per), c = (int)(i - (long long)r * per);
    const long long slot = (long long)len + r;
    if (slot >= C.cap()) continue;
    const long long o = C.row(b, slot, dh);
    const size_t src = (size_t)((long long)b * n + r) * (size_t)row_stride + (size_t)c * E;
    if (o >= 0 && (!mask || ((any >> r) & 1ull))) {
      *reinterpret_cast<uint4*>((T*)C.k + o + (long long)c * E) = __ldcg(reinterpret_cast<const uint4*>(k_new + src));
      *reinterpret_cast<uint4*>((T*)C.v + o + (long long)c * E) = __ldcg(reinterpret_cast<const uint4*>(v_new + src));
    }
    if (C.pos && (c * E) % dh == 0) {
      const size_t at = ((size_t)b * C.hkv + c * E / dh) * (size_t)C.cap() + (size_t)slot;
      C.pos[at] = C.seen[b] + r;
      C.weight[at] = 0.f;
    }
  }
}

// Keeps the accepted path of n uncommitted rows: slot len + acc_slot[j] moves to slot len + j, j < acc_len. acc_slot rises
// strictly and acc_slot[j] >= j, so a row's source is read before any row that could overwrite it is written when all of
// them are read first: one CTA per (sequence, head) holds the path's rows (n <= 64) in registers. Entries that do not rise end
// the path; a row from or to a page that the table does not have is skipped. The heads' CTAs read len, so its advance is a
// launch of its own (paged_advance_kernel).
template <typename T>
__global__ void __launch_bounds__(256) paged_path_kernel(PagedView C, int n, const int* acc_slot, const int* acc_len, int cap, int dh) {
  pdl_trigger();
  pdl_wait();
  constexpr int E = 16 / sizeof(T);
  const int h = blockIdx.x, b = blockIdx.y;
  const int len = C.len[b];
  if (len < 0) return;
  __shared__ int s_n, s_slot[64];
  if (threadIdx.x == 0) {
    int m = min(min(acc_len[b], cap), n), last = -1, j = 0;
    for (; j < m; ++j) {
      const int s = acc_slot[(size_t)b * cap + j];
      if (s <= last || s >= n || (long long)len + s >= C.cap()) break;
      s_slot[j] = last = s;
    }
    s_n = j;
  }
  __syncthreads();
  const int m = s_n, per = dh / E;
  constexpr int MAXV = 64 * 32 / 256;                                // 16-byte pieces per thread: 64 rows x at most 32 pieces
  uint4 rk[MAXV], rv[MAXV];
#pragma unroll
  for (int u = 0; u < MAXV; ++u) {
    const int i = threadIdx.x + u * 256;
    const int j = i / per, c = i - j * per;
    if (j < m && s_slot[j] != j) {
      const long long o = C.row(b, (long long)len + s_slot[j], dh);
      if (o >= 0) {
        rk[u] = *reinterpret_cast<const uint4*>((const T*)C.k + o + (long long)h * dh + c * E);
        rv[u] = *reinterpret_cast<const uint4*>((const T*)C.v + o + (long long)h * dh + c * E);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < MAXV; ++u) {
    const int i = threadIdx.x + u * 256;
    const int j = i / per, c = i - j * per;
    if (j < m && s_slot[j] != j) {
      const long long from = C.row(b, (long long)len + s_slot[j], dh), o = C.row(b, (long long)len + j, dh);
      if (o >= 0 && from >= 0) {
        *reinterpret_cast<uint4*>((T*)C.k + o + (long long)h * dh + c * E) = rk[u];
        *reinterpret_cast<uint4*>((T*)C.v + o + (long long)h * dh + c * E) = rv[u];
      }
    }
  }
}

__global__ void __launch_bounds__(64) paged_advance_kernel(int* len, int* seen, int batch, int n, const int* acc_len, int n_rows, long long cap) {
  pdl_trigger();
  pdl_wait();
  const int b = threadIdx.x;
  if (b >= batch || len[b] < 0) return;
  const int add = max(0, min(acc_len ? acc_len[b] : n, n_rows));
  len[b] = (int)min((long long)len[b] + add, cap);
  if (seen) seen[b] += add;
}

}  // namespace moa
