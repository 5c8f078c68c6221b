// Attention of new rows over a paged key / value cache (sm_100a): one token per sequence, or the rows of a kept draft
// tree, against every cached position and the rows' own uncommitted slots.
//
//   s_j = scale * q . k_j,  p_j = exp(s_j - max s) / sum exp(s - max s),  out = sum_j p_j v_j
//
// What bounds it: one token reads every cached byte once for 4 * group multiply-adds per 4 bytes (bf16), so the cache
// stream from HBM does. The layout follows from that: the queries that share a key / value head -- (rows of the sequence)
// x (heads of the group) -- are stacked 16 to a tile, so a cached row is read once per 16 of them.
//
// Work split (paged_rows_kernel): the (sequence, head, query tile) items are laid end to end as tiles of positions, and
// the CTAs take equal consecutive stretches of that line, whatever the sequences' lengths are; the lengths are read on
// the device, so a captured graph follows them. A stretch may end inside an item: such an item is left in pieces
// (max, sum, unnormalised output) and paged_join_kernel adds them in the order of their positions, the same order on every
// run. Only the first and the last item of a stretch can be cut, so a CTA has two places for pieces: the first for the item
// its stretch begins in, the second for the one it ends in.
//
// Inside a CTA the four warps run on their own: each takes every fourth group of positions, keeps a three-stage ring of
// its own in shared memory (cp.async, no barrier of the CTA in the loop), and its own running maximum, sum and output; the
// four are merged once per item.
#pragma once
#include "moa_attn.cuh"

namespace moa {

constexpr int PG_WARPS = 4;
constexpr int PG_THREADS = PG_WARPS * 32;
constexpr int PG_STAGES = 3;
constexpr int PG_ROWS = 16;                  // query rows per tile
constexpr int PG_MAX_SEQ = 64;               // sequences per call
constexpr int PG_WAVES = 2;                  // CTAs per SM

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
  // element offset of (slot, head 0) of sequence b, or -1 where the table has no such page
  __device__ __forceinline__ long long row(int b, long long slot, int dh) const {
    const int page = __ldg(table + (size_t)b * max_pages + (size_t)(slot >> shift));
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
  float* whole_ml;                           // [items][PG_ROWS][2] of the items that were not cut, with score
  float* score; long long score_ld;          // [batch, hq, score_ld] scaled log2-domain scores, or null
  float* weight_out;                         // [batch, hkv, cap] or null
  int ctas;                                  // stretches the line is cut into at most
  int min_tiles;                             // ... and the least tiles of one
};

// The line of work. tiles_of(b) position tiles per item of sequence b; pre[b] = items' tiles before sequence b, per item.
struct PagedLine {
  long long pre[PG_MAX_SEQ + 1];
  int len[PG_MAX_SEQ];
  long long total;                           // tiles of the whole line
  int ctas;
};

// Every thread of the CTA calls it; ends with a barrier.
__device__ __forceinline__ void paged_line(PagedLine& L, const PagedAttn& P, int tile) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    long long own[2], sum = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = lane * 2 + u;
      const int len = b < P.c.batch ? P.c.len[b] : -1;
      if (b < PG_MAX_SEQ) L.len[b] = (int)min((long long)len, P.c.cap());
      const long long keys = len < 0 ? 0 : min((long long)len + P.n_new, P.c.cap());
      own[u] = (keys + tile - 1) / tile;
      sum += own[u];
    }
    long long inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    L.pre[lane * 2] = inc - sum;
    L.pre[lane * 2 + 1] = inc - sum + own[0];
    if (lane == 31) {
      L.pre[PG_MAX_SEQ] = inc;
      L.total = inc * P.c.hkv * P.tiles;
      const long long most = (L.total + P.min_tiles - 1) / P.min_tiles;
      L.ctas = (int)max(1ll, min((long long)P.ctas, most));
    }
  }
  __syncthreads();
}
__device__ __forceinline__ long long line_begin(const PagedLine& L, int cta) { return L.total * cta / L.ctas; }
// the CTA whose stretch holds tile x: the i with total*i/ctas <= x < total*(i+1)/ctas (rounded down)
__device__ __forceinline__ int line_owner(const PagedLine& L, long long x) { return (int)(((x + 1) * L.ctas - 1) / L.total); }

// One warp's running state over a 16-row query tile, merged over the CTA's warps at the end of an item.
// (max in the log2 domain, sum, output) of row r, all in fp32.

// ---------------------------------------------------------------------------------------------
// bf16: mma.sync m16n8k16, 16 positions per warp step. Scores and output accumulate in fp32. Probabilities enter the
// second product as two bf16 terms (hi + lo, 16 bits of mantissa): rounding them once to 8 bits would put an error of up
// to 2^-9 of every term into the output, and the tensor pipe has room (48 products per 8 KB of cache).
// ---------------------------------------------------------------------------------------------
template <typename T, int DH> struct PagedWarp;

template <int DH>
struct PagedWarp<bf16, DH> {
  static constexpr int KW = 16;              // positions per warp step
  static constexpr int KS = DH / 16;
  uint32_t qf[KS][4];
  float o[DH / 8][4];
  float m[2], l[2];
  int gq, tq;

  __device__ __forceinline__ void start(const PagedAttn& P, int b, int h, int mt, uint8_t*) {
    const int lane = threadIdx.x & 31;
    gq = lane >> 2; tq = lane & 3;
    const int R = P.n * P.group;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = mt * PG_ROWS + gq + 8 * u;
      const bool in = r < R;
      const int rc = in ? r : 0;
      const uint32_t* src = reinterpret_cast<const uint32_t*>((const bf16*)P.q + ((long long)b * P.n + rc / P.group) * P.q_stride +
                                                              (long long)(h * P.group + rc % P.group) * DH);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint32_t x = __ldg(src + ks * 8 + tq), y = __ldg(src + ks * 8 + 4 + tq);
        qf[ks][u] = in ? x : 0u;
        qf[ks][2 + u] = in ? y : 0u;
      }
    }
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }

  // One step: 16 positions from `base` on, keys at sK, values at sV. live: bit per position that exists; see(u, j): whether
  // row u of this thread sees position j of the step; plain: every row sees every position.
  template <typename See>
  __device__ __forceinline__ void step(const PagedAttn& P, uint32_t sK, uint32_t sV, bool plain, See see, float* score0, float* score1) {
    const int lane = threadIdx.x & 31;
    float s[2][2][4];                        // [chain][8 positions][fragment]: two chains halve the products' latency
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) s[c][nt][0] = s[c][nt][1] = s[c][nt][2] = s[c][nt][3] = 0.f;
#pragma unroll
    for (int ks2 = 0; ks2 < KS / 2; ++ks2) {
      uint32_t kb[2][4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
        ldsm_x4(sK + tile_off<DH>(nt * 8 + (lane & 7), ks2 * 4 + (lane >> 3)), kb[nt][0], kb[nt][1], kb[nt][2], kb[nt][3]);
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) mma_bf16_16816(s[0][nt], qf[2 * ks2], kb[nt][0], kb[nt][1]);
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) mma_bf16_16816(s[1][nt], qf[2 * ks2 + 1], kb[nt][2], kb[nt][3]);
    }
    float z[2][4];                           // [row u][position nt*8 + 2*tq + e] = z[u][nt*2 + e]
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e >> 1][nt * 2 + (e & 1)] = (s[0][nt][e] + s[1][nt][e]) * P.scale_log2;
    if (!plain) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!see(u, (i >> 1) * 8 + 2 * tq + (i & 1))) z[u][i] = -INFINITY;
    }
    if (score0) {                            // the row's scores, for the accumulated weights
      *reinterpret_cast<float2*>(score0 + 2 * tq) = make_float2(z[0][0], z[0][1]);
      *reinterpret_cast<float2*>(score0 + 8 + 2 * tq) = make_float2(z[0][2], z[0][3]);
    }
    if (score1) {
      *reinterpret_cast<float2*>(score1 + 2 * tq) = make_float2(z[1][0], z[1][1]);
      *reinterpret_cast<float2*>(score1 + 8 + 2 * tq) = make_float2(z[1][2], z[1][3]);
    }
    float f[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float mx = fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float mn = fmaxf(m[u], mx);
      f[u] = (mn == m[u]) ? 1.f : ex2_approx(m[u] - mn);          // m = -inf: 0
      m[u] = mn;
    }
    if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) { o[i][0] *= f[0]; o[i][1] *= f[0]; o[i][2] *= f[1]; o[i][3] *= f[1]; }
      l[0] *= f[0];
      l[1] *= f[1];
    }
    uint32_t hi[4], lo[4];                   // A operand: rows gq, gq + 8 x positions 0..7, 8..15
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float sub = m[u] == -INFINITY ? 0.f : m[u];           // a row that has seen nothing: exp2(-inf - 0) = 0
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        const float p0 = ex2_approx(z[u][nt * 2] - sub), p1 = ex2_approx(z[u][nt * 2 + 1] - sub);
        l[u] += p0 + p1;
        const uint32_t w = pack_bf16(p0, p1);
        hi[nt * 2 + u] = w;
        lo[nt * 2 + u] = pack_bf16(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
      }
    }
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
      uint32_t v0, v1, v2, v3;               // values [16 positions x 16 columns] as two B fragments
      ldsm_x4_t(sV + tile_off<DH>(lane & 15, d * 2 + (lane >> 4)), v0, v1, v2, v3);
      mma_bf16_16816(o[2 * d], hi, v0, v1);
      mma_bf16_16816(o[2 * d + 1], hi, v2, v3);
      mma_bf16_16816(o[2 * d], lo, v0, v1);
      mma_bf16_16816(o[2 * d + 1], lo, v2, v3);
    }
  }

  // Leaves (max, sum) and the output of this warp's 16 rows in shared memory: so [16][DH], sml [16][2].
  __device__ __forceinline__ void finish(float* so, float* sml) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = l[u];
      t += __shfl_xor_sync(0xffffffffu, t, 1);
      t += __shfl_xor_sync(0xffffffffu, t, 2);
      const int r = gq + 8 * u;
      if (tq == 0) { sml[r * 2] = m[u]; sml[r * 2 + 1] = t; }
#pragma unroll
      for (int i = 0; i < DH / 8; ++i)
        *reinterpret_cast<float2*>(so + r * DH + i * 8 + 2 * tq) = make_float2(o[i][2 * u], o[i][2 * u + 1]);
    }
  }
  __device__ __forceinline__ int row_of(int u) const { return gq + 8 * u; }
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
  float m[PG_ROWS / 8], l[PG_ROWS / 8];      // lane's rows for the statistics: lane / 8 ... see step()
  float *sq, *sp;                            // queries [16][DH] of the CTA, this warp's probabilities [8][16]
  int rows;

  // Shared memory behind the rings: queries of the item [16][DH], then per warp probabilities [KW][PG_ROWS] and factors [16].
  static constexpr int SMEM = (PG_ROWS * DH + PG_WARPS * (KW + 1) * PG_ROWS) * 4;

  float mrow, lrow;                          // running max and sum of row (lane & 15); both half-warps hold the same

  __device__ __forceinline__ void start(const PagedAttn& P, int b, int h, int mt, uint8_t* extra) {
    const int R = P.n * P.group;
    sq = reinterpret_cast<float*>(extra);
    sp = sq + PG_ROWS * DH + (threadIdx.x >> 5) * (KW + 1) * PG_ROWS;
    rows = min(PG_ROWS, R - mt * PG_ROWS);
    for (int i = threadIdx.x; i < PG_ROWS * DH / 4; i += PG_THREADS) {
      const int rl = i / (DH / 4), c = i - rl * (DH / 4);
      const int r = mt * PG_ROWS + rl;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < R)
        x = __ldg(reinterpret_cast<const float4*>((const float*)P.q + ((long long)b * P.n + r / P.group) * P.q_stride +
                                                  (long long)(h * P.group + r % P.group) * DH) + c);
      reinterpret_cast<float4*>(sq)[i] = x;
    }
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r)
#pragma unroll
      for (int d = 0; d < DL; ++d) o[r][d] = 0.f;
    mrow = -INFINITY;
    lrow = 0.f;
    __syncthreads();
  }

  // 16-byte chunk of a row, swizzled by the row
  static __device__ __forceinline__ uint32_t off(int row, int chunk) { return (uint32_t)(row * (DH * 4) + ((chunk ^ (row & 7)) << 4)); }

  template <typename See>
  __device__ __forceinline__ void step(const PagedAttn& P, const uint8_t* K, const uint8_t* V, bool plain, See see, float* score, long long score_ld) {
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
      if (quarter == (r & 3)) sp[kk * PG_ROWS + r] = (plain || see(r, kk)) ? t * P.scale_log2 : -INFINITY;
    }
    __syncwarp();
    // softmax statistics: lane r of each half-warp holds row r
    {
      const int r = lane & 15;
      float z[KW], mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        z[k] = r < rows ? sp[k * PG_ROWS + r] : -INFINITY;
        mx = fmaxf(mx, z[k]);
      }
      if (score && lane < 16 && r < rows) {
#pragma unroll
        for (int k = 0; k < KW; k += 4) *reinterpret_cast<float4*>(score + r * score_ld + k) = make_float4(z[k], z[k + 1], z[k + 2], z[k + 3]);
      }
      const float mn = fmaxf(mrow, mx);
      const float f = mn == mrow ? 1.f : exp2f(mrow - mn);
      mrow = mn;
      const float sub = mn == -INFINITY ? 0.f : mn;
      lrow *= f;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float p = exp2f(z[k] - sub);
        lrow += p;
        if (lane < 16) sp[k * PG_ROWS + r] = p;
      }
      if (lane < 16) sp[KW * PG_ROWS + r] = f;
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

  __device__ __forceinline__ void finish(float* so, float* sml) {
    const int lane = threadIdx.x & 31;
    if (lane < 16) { sml[lane * 2] = mrow; sml[lane * 2 + 1] = lrow; }
#pragma unroll
    for (int r = 0; r < PG_ROWS; ++r)
#pragma unroll
      for (int d = 0; d < DL; ++d) so[r * DH + lane * DL + d] = o[r][d];
  }
};

template <typename T, int DH> struct PagedCfg {
  static constexpr int KW = PagedWarp<T, DH>::KW;
  static constexpr int TILE = PG_WARPS * KW;                    // positions per CTA step
  static constexpr int E = 16 / (int)sizeof(T);                 // elements per 16 bytes
  static constexpr int CH = DH / E;                             // 16-byte chunks per row
  static constexpr int ROW_BYTES = DH * (int)sizeof(T);
  static constexpr int HALF = KW * ROW_BYTES;                   // a warp's keys (or values) of one stage
  static constexpr int RING = PG_WARPS * PG_STAGES * 2 * HALF;
  static constexpr int MERGE = PG_WARPS * PG_ROWS * (DH + 2) * 4;     // lies over the rings
  static constexpr int EXTRA = sizeof(T) == 4 ? (PG_ROWS * DH + PG_WARPS * (8 + 1) * PG_ROWS) * 4 : 0;
  static constexpr int SMEM = (RING > MERGE ? RING : MERGE) + EXTRA;
};

// Union of the rows' masks: a new slot that no row sees is not read at all (what lies there may be anything).
__device__ __forceinline__ unsigned long long causal_word(int i) { return i >= 63 ? ~0ull : (2ull << i) - 1ull; }

template <typename T, int DH>
__global__ void __launch_bounds__(PG_THREADS, PG_WAVES) paged_rows_kernel(const PagedAttn P) {
  using C = PagedCfg<T, DH>;
  pdl_trigger();
  extern __shared__ __align__(128) uint8_t pg_smem[];
  __shared__ PagedLine L;
  __shared__ unsigned long long row_mask[64];
  __shared__ unsigned int live_of[PG_WARPS][PG_STAGES];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const extra = pg_smem + (C::SMEM - C::EXTRA);
  uint8_t* const ring = pg_smem + warp * (PG_STAGES * 2 * C::HALF);
  const uint32_t ring_s = smem_u32(ring);
  pdl_wait(KID_ATTN);
  paged_line(L, P, C::TILE);
  if ((int)blockIdx.x >= L.ctas || L.total == 0) return;
  const long long x_end = line_begin(L, blockIdx.x + 1);
  const int hm_n = P.c.hkv * P.tiles;
  const int R = P.n * P.group;
  PagedWarp<T, DH> W;

  int b = 0;
  for (long long x = line_begin(L, blockIdx.x); x < x_end;) {
    while (x >= L.pre[b + 1] * hm_n) ++b;
    const long long T_b = L.pre[b + 1] - L.pre[b];
    const long long in_b = x - L.pre[b] * hm_n;
    const int hm = (int)(in_b / T_b);
    const int h = hm / P.tiles, mt = hm - h * P.tiles;
    const long long t0 = in_b - hm * T_b, t1 = min(T_b, t0 + (x_end - x));
    const int len = L.len[b];
    const long long keys = min((long long)len + P.n_new, P.c.cap());

    // masks of the sequence's rows; any: some row sees the slot
    unsigned long long any = 0ull;
    bool full_rows = true;                                           // every row sees the committed slots
    if (P.mask) {
      if (threadIdx.x < P.n) row_mask[threadIdx.x] = P.mask[(size_t)b * P.n + threadIdx.x];
      __syncthreads();
      for (int i = 0; i < P.n; ++i) { any |= row_mask[i]; full_rows = full_rows && row_mask[i] != 0ull; }
    } else {
      any = causal_word(P.n - 1);
    }
    W.start(P, b, h, mt, extra);

    const int ch = lane % C::CH, r_first = lane / C::CH;
    constexpr int R_STEP = 32 / C::CH;
    // A step's rows -> this warp's ring. A row that does not exist is zero-filled: zero times what lies there may not be zero.
    auto issue = [&](long long t, int st) {
      const long long base = t * C::TILE + warp * C::KW;
      const uint32_t dK = ring_s + st * 2 * C::HALF, dV = dK + C::HALF;
      long long off = 0;
      int src = 0;                                                   // 0: does not exist, 1: page, 2: new row
      const long long key = base + lane;
      if (lane < C::KW && key < keys) {
        if (key >= len && !((any >> (key - len)) & 1ull)) {
          src = 0;
        } else if (key >= len && P.k_new) {
          src = 2;
          off = ((long long)b * P.n + (key - len)) * P.new_stride + (long long)h * DH;
        } else {
          off = P.c.row(b, key, DH);
          src = off >= 0 ? 1 : 0;
          off += (long long)h * DH;
        }
      }
      const unsigned live = __ballot_sync(0xffffffffu, src != 0);
      const unsigned fresh = __ballot_sync(0xffffffffu, src == 2);
      if (lane == 0) live_of[warp][st] = live;
      for (int r = r_first; r < C::KW; r += R_STEP) {
        const long long o = __shfl_sync(0xffffffffu, off, r);
        const bool ok = (live >> r) & 1u, nw = (fresh >> r) & 1u;
        const T* kp = (const T*)(nw ? P.k_new : P.c.k) + (ok ? o : 0) + ch * C::E;
        const T* vp = (const T*)(nw ? P.v_new : P.c.v) + (ok ? o : 0) + ch * C::E;
        const uint32_t d = (uint32_t)(r * C::ROW_BYTES + ((ch ^ (r & 7)) << 4));
        cp_async16(dK + d, kp, ok);
        cp_async16(dV + d, vp, ok);
      }
    };
#pragma unroll
    for (int st = 0; st < PG_STAGES - 1; ++st) {
      if (t0 + st < t1) issue(t0 + st, st);
      cp_async_commit();
    }
    int st = 0;
    for (long long t = t0; t < t1; ++t) {
      {
        const int nst = st == 0 ? PG_STAGES - 1 : st - 1;            // the stage of the step before this one
        if (t + PG_STAGES - 1 < t1) issue(t + PG_STAGES - 1, nst);
        cp_async_commit();
      }
      cp_async_wait<PG_STAGES - 1>();
      __syncwarp();
      const long long base = t * C::TILE + warp * C::KW;
      const unsigned live = live_of[warp][st];
      if (live != 0u) {
        uint8_t* sK = ring + st * 2 * C::HALF;
        uint8_t* sV = sK + C::HALF;
        constexpr unsigned ALL = C::KW == 32 ? 0xffffffffu : (1u << C::KW) - 1u;
        const bool plain = live == ALL && base + C::KW <= len && full_rows;
        // whether query row r of the tile sees position base + j
        auto sees = [&](int r, int j) -> bool {
          const int rr = mt * PG_ROWS + r;
          if (rr >= R || !((live >> j) & 1u)) return false;
          const int i = rr / P.group;
          const unsigned long long w = P.mask ? row_mask[i] : causal_word(i);
          const long long key = base + j;
          return key < len ? w != 0ull : ((w >> (key - len)) & 1ull) != 0ull;
        };
        if constexpr (sizeof(T) == 2) {
          float *s0 = nullptr, *s1 = nullptr;
          if (P.score) {                                             // one token: row = head of the group
            const int r0 = mt * PG_ROWS + W.row_of(0), r1 = mt * PG_ROWS + W.row_of(1);
            float* at = P.score + ((long long)b * P.hq + h * P.group) * P.score_ld + base;
            if (r0 < R) s0 = at + r0 * P.score_ld;
            if (r1 < R) s1 = at + r1 * P.score_ld;
          }
          W.step(P, smem_u32(sK), smem_u32(sV), plain, [&](int u, int j) { return sees(W.row_of(u), j); }, s0, s1);
        } else {
          float* at = P.score ? P.score + ((long long)b * P.hq + h * P.group + mt * PG_ROWS) * P.score_ld + base : nullptr;
          W.step(P, sK, sV, plain, sees, at, P.score_ld);
        }
        // the item's first query tile writes the new rows it holds to their pages
        if (P.k_new && mt == 0 && base + C::KW > len) {
          for (int r = r_first; r < C::KW; r += R_STEP) {
            const long long key = base + r;
            if (key < len || key >= keys || !((live >> r) & 1u)) continue;
            const long long o = P.c.row(b, key, DH);
            if (o < 0) continue;
            const uint32_t d = (uint32_t)(r * C::ROW_BYTES + ((ch ^ (r & 7)) << 4));
            *reinterpret_cast<uint4*>((T*)P.c.k + o + (long long)h * DH + ch * C::E) = *reinterpret_cast<const uint4*>(sK + d);
            *reinterpret_cast<uint4*>((T*)P.c.v + o + (long long)h * DH + ch * C::E) = *reinterpret_cast<const uint4*>(sV + d);
          }
        }
        __syncwarp();
      } else if (P.score) {                                          // nothing there: the weights' pass reads -inf
        for (int i = lane; i < C::KW * min(PG_ROWS, R - mt * PG_ROWS); i += 32)
          P.score[((long long)b * P.hq + h * P.group + mt * PG_ROWS + i / C::KW) * P.score_ld + base + i % C::KW] = -INFINITY;
      }
      if (P.k_new && mt == 0 && P.c.pos && base + C::KW > len && lane < C::KW) {
        const long long key = base + lane;
        if (key >= len && key < keys) {
          const size_t at = ((size_t)b * P.c.hkv + h) * (size_t)P.c.cap() + (size_t)key;
          P.c.pos[at] = P.c.seen[b] + (int)(key - len);
          P.c.weight[at] = 0.f;
        }
      }
      st = st == PG_STAGES - 1 ? 0 : st + 1;
    }
    cp_async_wait<0>();
    __syncthreads();                                                 // the rings are free: the merge lies over them
    float* so = reinterpret_cast<float*>(pg_smem);                   // [warp][16][DH]
    float* sml = so + PG_WARPS * PG_ROWS * DH;                       // [warp][16][2]
    W.finish(so + warp * PG_ROWS * DH, sml + warp * PG_ROWS * 2);
    __syncthreads();
    const bool whole = t0 == 0 && t1 == T_b;
    const size_t piece = (size_t)blockIdx.x * 2 + (x == line_begin(L, blockIdx.x) ? 0 : 1);
    float* const ml_at = whole ? (P.score ? P.whole_ml + ((size_t)b * hm_n + hm) * PG_ROWS * 2 : nullptr) : P.part_ml + piece * PG_ROWS * 2;
    for (int i = threadIdx.x; i < PG_ROWS * (DH / 4); i += PG_THREADS) {
      const int r = i / (DH / 4), c = i - r * (DH / 4);
      const int rr = mt * PG_ROWS + r;
      if (rr >= R) break;
      float mw[PG_WARPS], M = -INFINITY;
#pragma unroll
      for (int w = 0; w < PG_WARPS; ++w) { mw[w] = sml[(w * PG_ROWS + r) * 2]; M = fmaxf(M, mw[w]); }
      const float sub = M == -INFINITY ? 0.f : M;
      float S = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < PG_WARPS; ++w) {
        const float f = exp2f(mw[w] - sub);
        S = fmaf(f, sml[(w * PG_ROWS + r) * 2 + 1], S);
        const float4 y = *reinterpret_cast<const float4*>(so + (w * PG_ROWS + r) * DH + c * 4);
        a.x = fmaf(f, y.x, a.x); a.y = fmaf(f, y.y, a.y); a.z = fmaf(f, y.z, a.z); a.w = fmaf(f, y.w, a.w);
      }
      if (whole) {
        if (S == 0.f) a = make_float4(0.f, 0.f, 0.f, 0.f);           // the row sees nothing
        const float inv = S == 0.f ? 0.f : 1.f / S;                  // a NaN stays one
        T* dst = (T*)P.out + (((size_t)b * P.n + rr / P.group) * P.hq + h * P.group + rr % P.group) * DH + c * 4;
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
        else
          *reinterpret_cast<float4*>(dst) = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
      } else {
        *reinterpret_cast<float4*>(P.part_o + (piece * PG_ROWS + r) * DH + c * 4) = a;
      }
      if (c == 0 && ml_at) {
        ml_at[r * 2] = M;
        ml_at[r * 2 + 1] = S;
      }
    }
    x += t1 - t0;
    __syncthreads();                                                 // the merge is read before the rings fill again
  }
}

// The piece that CTA c holds of an item that begins at x0: its first place unless the item begins inside its stretch.
__device__ __forceinline__ size_t piece_of(const PagedLine& L, int c, long long x0) { return (size_t)c * 2 + (line_begin(L, c) >= x0 ? 0 : 1); }

// Joins the pieces of the items that a stretch's end cut, in the order of their positions; rows of sequences without any
// position become zero. Work: every end of a stretch times the rows of an item (ROWS), each for NW warps of a CTA that take
// every NW-th piece and add their sums in warp order; an item that several ends cut belongs to the first of them. Then the
// weights: weight_out = weight + sum over the group's heads of exp2(score - max) / sum, slots 0 .. keys - 1, 256 slots per CTA
// at a time.
template <typename T, int DH, int ROWS, int NW>
__global__ void __launch_bounds__(128) paged_join_kernel(const PagedAttn P, int tile) {
  pdl_trigger();
  __shared__ PagedLine L;
  __shared__ float s_m[128], s_l[128];
  __shared__ float s_o[4][DH + 1];
  pdl_wait(KID_ATTN_MERGE);
  paged_line(L, P, tile);
  const int hm_n = P.c.hkv * P.tiles, R = P.n * P.group;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int DL = DH / 32, UNITS = 4 / NW;              // rows that a CTA joins side by side
  const int sub = warp / NW, wq = warp % NW;
  const long long n_units = (long long)(L.total > 0 ? L.ctas - 1 : 0) * ROWS;
  for (long long w0 = (long long)blockIdx.x * UNITS; w0 < n_units; w0 += (long long)gridDim.x * UNITS) {
    const long long w = w0 + sub;
    const int c = (int)(w / ROWS) + 1, r = (int)(w % ROWS);
    const long long x = w < n_units ? line_begin(L, c) : 0;
    int b = 0, hm = 0;
    long long x0 = 0, T_b = 1;
    bool todo = w < n_units;
    if (todo) {
      int hi = PG_MAX_SEQ;                                 // the sequence that holds tile x: pre[b] * hm_n <= x < pre[b + 1] * hm_n
      while (hi - b > 1) {
        const int mid = (b + hi) >> 1;
        if (L.pre[mid] * hm_n <= x) b = mid; else hi = mid;
      }
      T_b = L.pre[b + 1] - L.pre[b];
      hm = (int)((x - L.pre[b] * hm_n) / T_b);
      x0 = L.pre[b] * hm_n + hm * T_b;
      todo = x != x0 && line_owner(L, x0) == c - 1 && hm % P.tiles * ROWS + r < R;
    }
    float S = 0.f, a[DL];
#pragma unroll
    for (int d = 0; d < DL; ++d) a[d] = 0.f;
    if (todo) {
      const int c1 = line_owner(L, x0 + T_b - 1);
      float M = -INFINITY;
      for (int i = c - 1 + lane; i <= c1; i += 32) M = fmaxf(M, P.part_ml[(piece_of(L, i, x0) * ROWS + r) * 2]);
      M = warp_max(M);
      const float ref = M == -INFINITY ? 0.f : M;
      for (int i = c - 1 + wq; i <= c1; i += NW) {
        const size_t at = piece_of(L, i, x0) * ROWS + r;
        const float f = exp2f(P.part_ml[at * 2] - ref);
        S = fmaf(f, P.part_ml[at * 2 + 1], S);
#pragma unroll
        for (int d = 0; d < DL; ++d) a[d] = fmaf(f, P.part_o[at * DH + lane * DL + d], a[d]);
      }
    }
    if constexpr (NW > 1) {
      __syncthreads();
      if (wq > 0) {
#pragma unroll
        for (int d = 0; d < DL; ++d) s_o[warp][lane * DL + d] = a[d];
        if (lane == 0) s_o[warp][DH] = S;
      }
      __syncthreads();
      if (wq == 0) {
        for (int k = 1; k < NW; ++k) {
#pragma unroll
          for (int d = 0; d < DL; ++d) a[d] += s_o[warp + k][lane * DL + d];
          S += s_o[warp + k][DH];
        }
      }
    }
    if (todo && wq == 0) {
      const int rr = hm % P.tiles * ROWS + r;
      T* dst = (T*)P.out + (((size_t)b * P.n + rr / P.group) * P.hq + hm / P.tiles * P.group + rr % P.group) * DH + lane * DL;
      const float inv = S == 0.f ? 0.f : 1.f / S;
#pragma unroll
      for (int d = 0; d < DL; ++d) dst[d] = from_f<T>(S == 0.f ? 0.f : a[d] * inv);
    }
  }
  for (int b = blockIdx.x; b < P.c.batch; b += gridDim.x) {
    if (L.len[b] < 0 || L.pre[b + 1] != L.pre[b]) continue;
    T* dst = (T*)P.out + (size_t)b * P.n * P.hq * DH;
    for (int d = threadIdx.x; d < P.n * P.hq * DH; d += 128) dst[d] = from_f<T>(0.f);
  }
  if (!P.weight_out) return;
  // weights: chunks of 256 slots of every (sequence, head), counted along the lengths
  constexpr int CHUNK = 256;
  long long n_chunks = 0;
  for (int b = 0; b < P.c.batch; ++b)
    if (L.len[b] >= 0) n_chunks += ((min((long long)L.len[b] + P.n_new, P.c.cap()) + CHUNK - 1) / CHUNK) * P.c.hkv;
  long long base = 0;
  int b = -1;
  long long per = 0;
  for (long long w = blockIdx.x; w < n_chunks; w += gridDim.x) {
    while (b < 0 || w >= base + per * P.c.hkv) {
      if (b >= 0) base += per * P.c.hkv;
      ++b;
      per = L.len[b] < 0 ? 0 : (min((long long)L.len[b] + P.n_new, P.c.cap()) + CHUNK - 1) / CHUNK;
    }
    const int h = (int)((w - base) / per);
    const long long slot0 = (w - base - h * per) * CHUNK;
    const long long keys = min((long long)L.len[b] + P.n_new, P.c.cap());
    const long long T_b = L.pre[b + 1] - L.pre[b];
    __syncthreads();
    for (int g = threadIdx.x; g < P.group; g += 128) {              // the heads' maximum and sum over their pieces
      const int hm = h * P.tiles + g / PG_ROWS, r = g % PG_ROWS;
      const long long x0 = L.pre[b] * hm_n + (long long)hm * T_b;
      const int c0 = line_owner(L, x0), c1 = line_owner(L, x0 + T_b - 1);
      float M = -INFINITY, S = 0.f, sub;
      if (c0 == c1) {
        const float* ml = P.whole_ml + (((size_t)b * hm_n + hm) * PG_ROWS + r) * 2;
        M = ml[0];
        S = ml[1];
        sub = M == -INFINITY ? 0.f : M;
      } else {
        for (int i = c0; i <= c1; ++i) M = fmaxf(M, P.part_ml[(piece_of(L, i, x0) * PG_ROWS + r) * 2]);
        sub = M == -INFINITY ? 0.f : M;
        for (int i = c0; i <= c1; ++i) {
          const float* ml = P.part_ml + (piece_of(L, i, x0) * PG_ROWS + r) * 2;
          S = fmaf(exp2f(ml[0] - sub), ml[1], S);
        }
      }
      s_m[g] = sub;
      s_l[g] = S == 0.f ? 0.f : 1.f / S;
    }
    __syncthreads();
    for (long long slot = slot0 + threadIdx.x; slot < min(slot0 + CHUNK, keys); slot += 128) {
      const size_t at = ((size_t)b * P.c.hkv + h) * (size_t)P.c.cap() + (size_t)slot;
      float sum = 0.f;
      const float* s = P.score + ((long long)b * P.hq + h * P.group) * P.score_ld + slot;
      for (int g = 0; g < P.group; ++g) sum = fmaf(exp2f(s[g * P.score_ld] - s_m[g]), s_l[g], sum);
      const float old = (P.c.weight && slot < L.len[b]) ? P.c.weight[at] : 0.f;
      P.weight_out[at] = old + sum;
    }
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
    for (int i = 0; i < n; ++i) any |= __ldg(mask + (size_t)b * n + i);
  }
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)rows * per; i += (long long)gridDim.x * blockDim.x) {
    const int r = (int)(i / per), c = (int)(i - (long long)r * per);
    const long long slot = (long long)len + r;
    if (slot >= C.cap()) continue;
    const long long o = C.row(b, slot, dh);
    const size_t src = (size_t)((long long)b * n + r) * (size_t)row_stride + (size_t)c * E;
    if (o >= 0 && (!mask || ((any >> r) & 1ull))) {
      *reinterpret_cast<uint4*>((T*)C.k + o + (long long)c * E) = __ldg(reinterpret_cast<const uint4*>(k_new + src));
      *reinterpret_cast<uint4*>((T*)C.v + o + (long long)c * E) = __ldg(reinterpret_cast<const uint4*>(v_new + src));
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
// them are read first: one CTA per (sequence, head) holds the path's rows (cap <= 64) in registers. Entries that do not
// rise end the path. Then len (and seen) advance, when asked to, by one thread of the sequence's first CTA -- the heads'
// CTAs read len, so the advance is a launch of its own.
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
