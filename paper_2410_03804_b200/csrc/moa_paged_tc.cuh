// Attention of many query rows per key / value head over a paged cache, on the 5th-generation tensor cores (sm_100a, bf16):
// the rows of a kept draft tree (up to 64 rows x the heads of a group).
//
// With 244 rows (61 slots, group 4) a cached byte takes part in 244 multiply-adds, so the tensor pipe and the exponentials
// bound it, not HBM: per 128 positions and 128 rows two products of 128 x 128 x 128 (512 cycles each at the pipe's rate) and
// 16384 exponentials (1024 cycles at 16 a cycle and SM). Two query tiles of 128 rows share one stream of keys and values and
// take turns: while one tile's scores become probabilities in registers, the pipe works on the other tile.
//   warp 0      copies: keys and values of 128 positions per ring slot (32 KB at head size 128, five slots, K V K V ...), by TMA
//               page by page: box [page rows, 64 columns], 128-byte swizzle; a page that the table does not have, or that
//               lies behind the last position, is asked for behind the pool's end and arrives as zeros
//   warp 1      tcgen05.mma: S_i = Q_i K^T (Q in shared memory), O_i += P_i V (P in tensor memory, V as it lies in the
//               cache: MN-major)
//   warps 2..5  softmax of tile 0, one thread per query row; warps 6..9 of tile 1. P_i goes over S_i in tensor memory.
// Blocks of 64 positions with two score buffers per tile were tried: nothing waits for a tile's own products then, but a
// product costs about 60 cycles at N = 64 as at N = 128, and the pipe was the limit (4700 cycles per 128 positions).
// Tensor memory: S_0 S_1 O_0 O_1, 128 columns each. The output is rescaled only when a row's maximum grew by more than 2^8.
// The probabilities enter the second product rounded once to bf16 (each off by at most 2^-8 of itself, so an output is off by
// at most 2^-8 * sum p |v|, the size of its own rounding to bf16), while their sum is taken in fp32 before the rounding. With two
// terms, as in the row kernel, the error against 64 bits fell from 0.0023 to 0.0017 of the output (its rounding alone) and the
// large case below went from 173 to 211 us, 204 to 245 over seconds.
// Work split and pieces are those of the row kernel, with items of 256 query rows and one CTA per SM; the pieces are joined by
// a kernel behind it (paged_join_kernel), whose CTAs are four per cut item: the 128 KB of an item are too much for one.
// Measured: 16 sequences x 61 rows x 64 heads over 4096 positions (0.133 TFLOP of products, 0.27 GB of cache): 173 us in short
// bursts of replays, 198 to 204 us over seconds of calls (0.65 to 0.67 PFLOP/s without the padding to 512 rows). With half the
// sequences the counters show the tensor pipe and the exponential unit at 40 % each and 1.05 instructions a cycle and SM: neither
// pipe is the limit, but the chain of one block -- score product, one thread's pass over its row of 128 scores, output product --
// of which two tiles are under way. 61 rows x 32 heads over 2048 positions: 29 us, two thirds of it the start (tensor memory,
// table, first copies: 9 us) and the join. The row kernel took 1537 and 44 us for the two.
// Every wait is bounded; a CTA whose wait ran out writes NaN to its rows (the serving calls have no status word).
#pragma once
#include "moa_attn_tc.cuh"
#include "moa_paged.cuh"

namespace moa {

constexpr int PT_KB = 128;                   // positions per block
constexpr int PT_ROWS = 256;                 // query rows per item: two tiles
constexpr int PT_THREADS = 320;
constexpr int PT_SLOTS = 5;
constexpr uint32_t PT_TM_S = 0, PT_TM_O = 256;

template <int DH> struct PtCfg {
  static constexpr int CK = DH / 64;                          // 64-column chunks of a row
  static constexpr int QCHUNK = 128 * 128, QTILE = CK * QCHUNK;
  static constexpr int CHUNK = PT_KB * 128, SLOT = CK * CHUNK; // of a ring slot
  static constexpr int SMEM = 2 * QTILE + PT_SLOTS * SLOT + 1024 + 256;
};

// 16-byte piece of a query row in its tile: 64-column chunks of 128-byte rows, 128-byte swizzle.
__device__ __forceinline__ int pt_q_off(int row, int piece) { return (piece >> 3) * (128 * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4); }

struct PagedTree {
  CUtensorMap tmK, tmV;                      // [n_pages, page_size, hkv * DH], box 64 columns x min(page_size, 128) rows
  PagedAttn a;
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
// Joins the pieces of the items that a stretch's end cut, in the order of their positions; an item that several ends cut
// belongs to the first of them, whose CTA has written down what it is. CTA (end of a stretch, quarter of the columns): a warp
// per 32 rows, a row per lane.
template <int DH>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedAttn P) {
  pdl_trigger();
  pdl_wait(KID_ATTN_MERGE);
  const int4 j0 = __ldcg(reinterpret_cast<const int4*>(P.joins) + blockIdx.x * 2), j1 = __ldcg(reinterpret_cast<const int4*>(P.joins) + blockIdx.x * 2 + 1);
  const int c = blockIdx.x + 1, c1 = j0.x, fp = j0.y, b = j0.z, h = j0.w, mt = j1.x;         // c1: last CTA with a piece, 0: no join
  if (c1 == 0) return;
  const int r = threadIdx.x, rr = mt * PT_ROWS + r;                  // row of the item, of the (sequence, head)
  const int R = P.n * P.group;
  if ((rr & ~31) >= R) return;
  float M = -INFINITY, Z = 0.f;
#pragma unroll 4
  for (int i = c - 1; i <= c1; ++i) M = fmaxf(M, __ldcg(P.part_ml + ((size_t)piece_of(i, c - 1, fp) * PT_ROWS + r) * 2));
  const float ref = M == -INFINITY ? 0.f : M;
  constexpr int N4 = DH / 16;                                        // 16-byte pieces of a row in a quarter
  float4 a[N4];
#pragma unroll
  for (int d = 0; d < N4; ++d) a[d] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int i = c - 1; i <= c1; ++i) {
    const size_t piece = piece_of(i, c - 1, fp);
    const float2 ml = __ldcg(reinterpret_cast<const float2*>(P.part_ml) + piece * PT_ROWS + r);
    const float f = exp2f((ml.x - ref) * P.scale_log2);
    Z = fmaf(f, ml.y, Z);
#pragma unroll
    for (int d = 0; d < N4; ++d) {
      const float4 o = __ldcg(reinterpret_cast<const float4*>(P.part_o) + (piece * (DH / 4) + blockIdx.y * N4 + d) * PT_ROWS + r);
      a[d].x = fmaf(f, o.x, a[d].x); a[d].y = fmaf(f, o.y, a[d].y); a[d].z = fmaf(f, o.z, a[d].z); a[d].w = fmaf(f, o.w, a[d].w);
    }
  }
  if (rr >= R) return;
  const float inv = Z == 0.f ? 0.f : 1.f / Z;
  bf16* dst = (bf16*)P.out + (((size_t)b * P.n + rr / P.group) * P.hq + h * P.group + rr % P.group) * DH + blockIdx.y * (DH / 4);
#pragma unroll
  for (int d = 0; d < N4; d += 2) {
    uint4 y = make_uint4(0u, 0u, 0u, 0u);
    if (Z != 0.f)
      y = make_uint4(pack_bf16(a[d].x * inv, a[d].y * inv), pack_bf16(a[d].z * inv, a[d].w * inv), pack_bf16(a[d + 1].x * inv, a[d + 1].y * inv),
                     pack_bf16(a[d + 1].z * inv, a[d + 1].w * inv));
    *reinterpret_cast<uint4*>(dst + d * 4) = y;
  }
}

// One stretch of an item, as every role of the CTA walks through them.
struct PtWalk {
  int x, x_begin, x_end;
  PagedPlace S;
  // the current segment
  int b, h, pair, t0, nb, x0;
  bool whole;
  __device__ __forceinline__ void begin(const PagedLine& L) {
    x = x_begin = L.x_begin;
    x_end = L.x_end;
    S = L.first;
  }
  __device__ __forceinline__ bool next(const PagedLine& L, const PagedAttn& P) {
    if (x >= x_end) return false;
    if (x != x_begin) S.at(L, P, x);
    b = S.b; h = S.h; pair = S.mt; t0 = S.t; x0 = x - t0;
    nb = min(S.T_b - t0, x_end - x);
    whole = nb == S.T_b;
    x += nb;
    return true;
  }
};

// Two fp32 values side by side (packed fp32 instructions of sm_100).
__device__ __forceinline__ uint64_t f2_pack(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ bool pt_elect() {               // one lane of a converged warp, the same one every time
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0u;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {      // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// bits of positions base .. base + 63 that a row with mask word w sees: committed ones (if it sees anything) and its new slots
__device__ __forceinline__ unsigned long long low_bits(long long n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }
__device__ __forceinline__ unsigned long long row_bits(unsigned long long w, long long base, int len, long long keys) {
  const long long s = len - base;
  unsigned long long v = w ? low_bits(s) : 0ull;
  if (s > -64 && s < 64) v |= s >= 0 ? w << s : w >> -s;
  return v & low_bits(keys - base);
}

// Rare steps of the softmax, kept out of its loop's code: inline they cost the loop 2 to 6 % without ever running.

// Probabilities of a block's scores (tensor memory, at tS), over the scores, for rows with scores far from zero; returns their sum.
__device__ __noinline__ float pt_steep(uint32_t tS, bool masked, unsigned long long vis0, unsigned long long vis1, float sub, float scale) {
  float l = 0.f;
#pragma unroll 1
  for (int e0 = 0; e0 < PT_KB; e0 += 16) {   // the probabilities, two to a column, stay behind the scores that are read
    float s[16];
    tc_ld16(tS + (uint32_t)e0, s);
    const uint32_t v = (uint32_t)((e0 < 64 ? vis0 : vis1) >> (e0 & 63));
    uint32_t w8[8];
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p0 = masked && !((v >> e) & 1u) ? 0.f : ex2_approx((s[e] - sub) * scale);
      const float p1 = masked && !((v >> e) & 2u) ? 0.f : ex2_approx((s[e + 1] - sub) * scale);
      l += p0 + p1;
      w8[e / 2] = pack_bf16(p0, p1);
    }
    tc_st8(tS + (uint32_t)(e0 / 2), w8);
  }
  return l;
}
// A row of a ring slot's values: cleared, or, where its position is there, cleared of what is not finite.
template <int DH>
__device__ __noinline__ void pt_clear(uint8_t* at, int row, bool there, volatile int* odd_flag) {
  auto piece = [&](int p) { return reinterpret_cast<uint4*>(at + (p >> 3) * PtCfg<DH>::CHUNK + (((p ^ row) & 7) << 4)); };
  if (!there) {
#pragma unroll
    for (int p = 0; p < DH / 8; ++p) *piece(p) = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  uint32_t top = 0u;                         // exponents of all ones carry into the signs
#pragma unroll
  for (int p = 0; p < DH / 8; ++p) {
    const uint4 x = *piece(p);
    top |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u);
    top |= ((x.z & 0x7f807f80u) + 0x00800080u) | ((x.w & 0x7f807f80u) + 0x00800080u);
  }
  if ((top & 0x80008000u) == 0u) return;
  *odd_flag = 1;
  __threadfence_block();                     // who finds the bytes cleared finds the flag
#pragma unroll 1
  for (int p = 0; p < DH / 8; ++p) *piece(p) = odd_cleared(*piece(p));
}
// Adds to a row's output (tensor memory, at tO) the values that are not finite of the new slots that it sees among positions
// from .. to - 1. A whole warp; the rows' words may differ.
template <int DH>
__device__ __noinline__ void pt_add_odd(const PagedAttn& P, int b, int h, long long from, long long to, int len, long long keys, unsigned long long word,
                                        uint32_t tO) {
  for (int d = 0; d < DH; d += 16) {
    float o[16];
    tc_ld16(tO + (uint32_t)d, o);
    for (int j = 0; j < P.n_new; ++j) {
      const long long key = (long long)len + j, at = key >= from && key < to && key < keys && ((word >> j) & 1ull) ? P.c.row(b, key, DH) : -1;
      if (at < 0) continue;
      const bf16* v = (const bf16*)P.c.v + at + (long long)h * DH + d;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = __bfloat162float(v[e]);
        if (odd_f(x)) o[e] += x;
      }
    }
    __syncwarp();
    tc_st16(tO + (uint32_t)d, o);
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

template <int DH>
__global__ void __launch_bounds__(PT_THREADS, 1) paged_tree_kernel(const __grid_constant__ PagedTree PP) {
  using C = PtCfg<DH>;
  extern __shared__ uint8_t pt_smem_raw[];
  __shared__ PagedLine L;
  const PagedAttn& P = PP.a;
  const uint32_t base = (smem_u32(pt_smem_raw) + 1023u) & ~1023u;
  uint8_t* bp = pt_smem_raw + (base - smem_u32(pt_smem_raw));
  const uint32_t oRing = 2 * C::QTILE, oBar = oRing + PT_SLOTS * C::SLOT, bar0 = base + oBar;
  auto slot_at = [&](uint32_t s) { return base + oRing + s * (uint32_t)C::SLOT; };
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (PT_SLOTS + s); };
  auto q_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + i); };
  auto o_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 2 + i); };
  auto s_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 4 + i); };
  auto p_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 6 + i); };
  uint32_t* tmem_slot = (uint32_t*)(bp + oBar + 8 * (2 * PT_SLOTS + 8));
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  volatile int* odd_flag = abort_flag + 1;   // a new slot's value that is not finite was met
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = P.n * P.group;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < PT_SLOTS; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_bar(i), 128);
      mbar_init(o_bar(i), 1);
      mbar_init(s_bar(i), 1);
      mbar_init(p_bar(i), 128);
    }
    *abort_flag = *odd_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait(KID_ATTN);
  paged_line(L, P, PT_KB);                   // ends with a barrier
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const bool idle = L.x_begin == L.x_end;
  PtWalk W;
  if (!idle) W.begin(L);

  if (idle) {
    if (threadIdx.x == 0) P.joins[blockIdx.x * 8] = 0;
  } else if (warp == 0) {
    // ------------------------------ copies ------------------------------
    const int rows = min(PT_KB, 1 << P.c.shift), sub_n = PT_KB / rows;        // rows of a box, boxes per chunk
    const int sub = lane % sub_n, chunk = lane / sub_n;
    const bool mine = lane < C::CK * sub_n;
    uint32_t cnt = 0;
    bool ok = true;
    while (ok && W.next(L, P)) {
      const long long keys = min((long long)L.len[W.b] + P.n_new, P.c.cap());
      const int* table = P.c.table + (size_t)W.b * P.c.max_pages;
      const int x0 = W.h * DH + chunk * 64;
      for (int t = 0; t < W.nb && ok; ++t) {
        const long long slot0 = (long long)(W.t0 + t) * PT_KB + sub * rows;
        int page = mine && slot0 < keys ? table[slot0 >> P.c.shift] : P.c.n_pages;
        if (page < 0 || page > P.c.n_pages) page = P.c.n_pages;
        const int y = (int)(slot0 & ((1 << P.c.shift) - 1));
        for (int kv = 0; kv < 2; ++kv, ++cnt) {
          const uint32_t s = cnt % PT_SLOTS;
          ok = mbar_wait(empty_bar(s), ((cnt / PT_SLOTS) & 1u) ^ 1u, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          // The first queries before the ring fills: together they are what the start waits for. Only inside the first
          // segment, which cannot end before this block comes: behind it the queries of the next one may have completed
          // the barrier's second phase, and the wait for the first would miss it.
          if (cnt == 2 && t == 1) {
            ok = mbar_wait(q_bar(0), 0u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
          }
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(full_bar(s), C::SLOT);
          __syncwarp();
          if (mine) tma_load_3d(slot_at(s) + chunk * C::CHUNK + sub * rows * 128, kv ? &PP.tmV : &PP.tmK, x0, y, page, full_bar(s));
        }
      }
    }
    if (lane == 0) {                         // the item that the end of this stretch cuts first, for the join
      PagedPlace S;
      S.at(L, P, L.x_end - 1);
      const int x0 = L.x_end - 1 - S.t;
      int4* j = reinterpret_cast<int4*>(P.joins) + blockIdx.x * 2;
      const bool cut = x0 >= L.x_begin && x0 + S.T_b > L.x_end;
      j[0] = make_int4(cut ? line_owner(L, x0 + S.T_b - 1) : 0, x0 > L.x_begin ? 1 : 0, S.b, S.h);
      j[1] = make_int4(S.mt, 0, 0, 0);
    }
    if (!ok && lane == 0) {                  // given up: the copies under way still land before the CTA ends
      const long long t_end = clock64() + WS_WAIT_CYCLES;
      for (uint32_t c = cnt > PT_SLOTS ? cnt - PT_SLOTS : 0; c < cnt; ++c)
        while (!mbar_test(full_bar(c % PT_SLOTS), (c / PT_SLOTS) & 1u) && clock64() < t_end) {}
    }
  } else if (warp == 1) {
    // ------------------------------ products ------------------------------
    // The whole warp walks the loops, so that addresses and descriptors stay in uniform registers; one elected lane issues.
    // (With all of it under one lane's branch every product waited for its descriptors to be moved there: 125 cycles.)
    constexpr uint32_t IDESC_S = umma_idesc_bf16(128, PT_KB);
    constexpr uint32_t IDESC_O = umma_idesc_bf16_bmn(128, DH);
    uint32_t g = 0, cq[2] = {0u, 0u}, c[2] = {0u, 0u};        // ring block of the segment's first block; queries, blocks of the tiles
    bool ok = true;
    const bool leader = pt_elect();
    auto scores = [&](int i, uint32_t blk, int tiles) -> bool {               // S_i of ring block blk
      const uint32_t n = 2 * blk, s = n % PT_SLOTS;
      if (!__all_sync(0xffffffffu, mbar_wait(full_bar(s), (n / PT_SLOTS) & 1u, abort_flag))) return false;
      tc_fence_after();
      const uint64_t kd = umma_desc_sw128(slot_at(s)), qd = umma_desc_sw128(base + i * C::QTILE);
      const uint32_t d = tmem + PT_TM_S + i * 128;
      if (leader) {
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
          const uint64_t o = (uint64_t)((ks >> 2) * (C::CHUNK / 16) + 2 * (ks & 3));
          tc_mma_bf16(d, qd + o, kd + o, IDESC_S, ks > 0 ? 1u : 0u);
        }
        tc_commit(s_bar(i));
        if (i == tiles - 1) tc_commit(empty_bar(s));
      }
      __syncwarp();
      return true;
    };
    while (ok && W.next(L, P)) {
      const int tiles = W.pair * PT_ROWS + 128 < R ? 2 : 1;
      for (int i = 0; i < tiles && ok; ++i) {
        ok = __all_sync(0xffffffffu, mbar_wait(q_bar(i), cq[i]++ & 1u, abort_flag));
        tc_fence_after();
        if (ok) ok = scores(i, g, tiles);
      }
      for (int t = 0; t < W.nb && ok; ++t, ++g) {
        const uint32_t n = 2 * g + 1, s = n % PT_SLOTS;
        for (int i = 0; i < tiles && ok; ++i) {
          ok = mbar_wait(p_bar(i), c[i]++ & 1u, abort_flag);
          if (ok && i == 0) ok = mbar_wait(full_bar(s), (n / PT_SLOTS) & 1u, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = umma_desc_mn_sw128(slot_at(s), C::CHUNK);
          const uint32_t d = tmem + PT_TM_O + i * 128, pa = tmem + PT_TM_S + i * 128;
          if (leader) {
#pragma unroll
            for (int ks = 0; ks < PT_KB / 16; ++ks)
              tc_mma_bf16_ta(d, pa + ks * 8, vd + (uint64_t)(ks * (2048 / 16)), IDESC_O, (t > 0 || ks > 0) ? 1u : 0u);
            tc_commit(o_bar(i));
            if (i == tiles - 1) tc_commit(empty_bar(s));
          }
          __syncwarp();
          if (t + 1 < W.nb) ok = scores(i, g + 1, tiles);       // over the probabilities just multiplied: the pipe keeps the order
        }
      }
    }
  } else {
    // ------------------------------ softmax ------------------------------
    const int i = (warp - 2) >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t tS = tmem + PT_TM_S + i * 128 + lane_addr, tO = tmem + PT_TM_O + i * 128 + lane_addr;
    uint32_t g = 0, c = 0;                   // blocks of the CTA, of this tile
    bool dead = false;
    while (W.next(L, P)) {
      if (W.pair * PT_ROWS + i * 128 >= R) { g += W.nb; continue; }           // the item has one tile
      const int rr = W.pair * PT_ROWS + i * 128 + row;
      const bool valid = rr < R;
      const int qi = valid ? rr / P.group : 0, hd = valid ? rr - qi * P.group : 0;
      const int len = L.len[W.b];
      const long long keys = min((long long)len + P.n_new, P.c.cap());
      // ---- queries into shared memory (the tile's last scores have been formed: this thread waited for them) ----
      // The segment's loads go out together, before the first is waited for: mask words, the first block's pages, queries.
      const int* table = P.c.table + (size_t)W.b * P.c.max_pages;
      const unsigned long long* mask = P.mask ? P.mask + (size_t)W.b * P.n : nullptr;
      unsigned long long word = mask ? mask[qi] : causal_word(qi);
      unsigned long long any = mask && lane < P.n ? mask[lane] : 0ull, any2 = mask && lane + 32 < P.n ? mask[lane + 32] : 0ull;
      // the page of a block that this lane looks at (blocks of up to 16 pages), loaded a block ahead
      auto page_at = [&](int t) -> int {
        const long long at = (long long)(W.t0 + t) * PT_KB + ((long long)lane << P.c.shift);
        return t < W.nb && (lane << P.c.shift) < PT_KB && at < keys ? table[at >> P.c.shift] : 0;
      };
      int page_next = page_at(0);
      // queries, coalesced: the warp's 32 rows, 32 * 8 / DH of them per instruction, into shared memory (the tile's last scores
      // have been formed: this thread waited for them); rows behind the last one hold some real row and are worked on, but
      // not written
      constexpr int PIECES = DH / 8, RPI = 32 / PIECES;
      const int piece = lane % PIECES;
      {
        const long long off = ((long long)W.b * P.n + qi) * P.q_stride + (long long)(W.h * P.group + hd) * DH;
        uint4 x[PIECES];
#pragma unroll
        for (int u = 0; u < PIECES; ++u)
          x[u] = __ldcg(reinterpret_cast<const uint4*>((const bf16*)P.q + __shfl_sync(0xffffffffu, off, u * RPI + lane / PIECES)) + piece);
#pragma unroll
        for (int u = 0; u < PIECES; ++u)
          *reinterpret_cast<uint4*>(bp + i * C::QTILE + pt_q_off(quad * 32 + u * RPI + lane / PIECES, piece)) = x[u];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        mbar_arrive(q_bar(i));
      }
      // ---- what the rows see ----
      any |= any2;
      any = mask ? ((unsigned long long)__reduce_or_sync(0xffffffffu, (unsigned)(any >> 32)) << 32) | __reduce_or_sync(0xffffffffu, (unsigned)any)
                 : causal_word(P.n - 1);
      if (!valid) word = 0ull;
      const bool all_rows = __all_sync(0xffffffffu, word != 0ull || !valid);
      float m_ref = -INFINITY, l_run = 0.f;
      for (int t = 0; t < W.nb; ++t, ++g, ++c) {
        if (!dead) dead = __any_sync(0xffffffffu, !mbar_wait(s_bar(i), c & 1u, abort_flag));
        if (dead) continue;
        tc_fence_after();
        const long long k0 = (long long)(W.t0 + t) * PT_KB;
        const unsigned bad = __ballot_sync(0xffffffffu, page_next < 0 || page_next >= P.c.n_pages);   // pages the table does not have
        page_next = page_at(t + 1);
        const bool masked = k0 + PT_KB > len || bad != 0u || !all_rows;
        unsigned long long vis[2] = {~0ull, ~0ull};
        if (masked) {
          vis[0] = row_bits(word, k0, len, keys);
          vis[1] = row_bits(word, k0 + 64, len, keys);
          unsigned long long live[2] = {row_bits(any, k0, len, keys), row_bits(any, k0 + 64, len, keys)};
          for (unsigned m = bad; m != 0u; m &= m - 1u) {
            const int at = (__ffs(m) - 1) << P.c.shift;              // the page's first position; pages of 128 rows and more: all
            const unsigned long long bits = low_bits(1ll << P.c.shift);
            if (at < 64) { vis[0] &= ~(bits << at); live[0] &= ~(bits << at); }
            if (at >= 64 || P.c.shift > 6) { vis[1] &= ~(bits << (at & 63)); live[1] &= ~(bits << (at & 63)); }
          }
          // Zero times what lies in a slot that does not exist may not be zero: such values are cleared, by the tile's 128
          // threads a row each, once they have landed. So are the values of new slots that are not finite; the rows that
          // see them get them at the segment's end. (The other tile clears the same bytes itself.)
          if (k0 + PT_KB > len || ~(live[0] & live[1]) != 0ull) {
            const uint32_t v = 2 * g + 1, vs = v % PT_SLOTS;
            dead = __any_sync(0xffffffffu, !mbar_wait(full_bar(vs), (v / PT_SLOTS) & 1u, abort_flag));
            if (dead) continue;
            const bool there = (((row < 64 ? live[0] : live[1]) >> (row & 63)) & 1ull) != 0ull;
            if (!there || k0 + row >= len) pt_clear<DH>(bp + oRing + vs * C::SLOT + row * 128, row, there, odd_flag);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
        }
        // The block's scores in two halves of 64, so that they stay in registers: the upper half for its maximum, the lower
        // half for its maximum and its probabilities, the upper half again (the probabilities, two to a column, lie over
        // the lower half's scores).
        float s[64];
        auto load_half = [&](int half) {
          tc_ld64(tS + half * 64, s);
          if (masked) {
            const unsigned long long v = half ? vis[1] : vis[0];
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (!((v >> e) & 1ull)) s[e] = -INFINITY;
          }
        };
        float m_blk = -INFINITY;
#pragma unroll
        for (int half = 1; half >= 0; --half) {
          load_half(half);
          float m4[4] = {m_blk, s[0], s[1], s[2]};
          m4[0] = max3_nan(m4[0], s[3], s[3]);
#pragma unroll
          for (int e = 4; e < 60; e += 8)
#pragma unroll
            for (int u = 0; u < 4; ++u) m4[u] = max3_nan(m4[u], s[e + 2 * u], s[e + 2 * u + 1]);
          m4[0] = max3_nan(m4[0], s[60], s[61]);
          m4[1] = max3_nan(m4[1], s[62], s[63]);
          m_blk = max3_nan(max3_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]);
        }
        float f = 1.f;
        if (m_ref == -INFINITY) {
          m_ref = m_blk;                     // nothing has been added for this row yet
        } else if ((m_blk - m_ref) * P.scale_log2 > TC_RESCALE_LOG2) {
          f = ex2_approx((m_ref - m_blk) * P.scale_log2);
          m_ref = m_blk;
          l_run *= f;
        }
        if (t > 0 && __any_sync(0xffffffffu, f != 1.f)) {
          // rare: the output moves to a new reference; the last product must have left the tensor pipe
          dead = __any_sync(0xffffffffu, !mbar_wait(o_bar(i), (c - 1u) & 1u, abort_flag));
          if (dead) continue;
          tc_fence_after();
#pragma unroll 1
          for (int d = 0; d < DH; d += 16) {
            float o[16];
            tc_ld16(tO + (uint32_t)d, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= f;
            tc_st16(tO + (uint32_t)d, o);
          }
        }
        const float sub = m_ref == -INFINITY ? 0.f : m_ref;
        // scale * (score - reference) as one multiply-add, score * scale - (scale * reference). The latter is a rounded product,
        // half a unit of its last place off: the row's common factor, below 2^0.5 while it is below 2^24. From there on (or
        // where it leaves fp32) the difference is taken first.
        const float scaled = __fmul_rn(sub, P.scale_log2);
        if (__any_sync(0xffffffffu, fabsf(scaled) >= 16777216.f)) {
          l_run += pt_steep(tS, masked, vis[0], vis[1], sub, P.scale_log2);
        } else {
          const uint64_t scale2 = f2_pack(P.scale_log2, P.scale_log2), sub2 = f2_pack(-scaled, -scaled);
          uint64_t l2[2] = {0ull, 0ull};
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (half) load_half(1);
#pragma unroll
            for (int e = 0; e < 64; e += 16) {
              uint32_t w8[8];
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                float p0, p1;
                f2_unpack(f2_fma(f2_pack(s[e + 2 * u], s[e + 2 * u + 1]), scale2, sub2), p0, p1);
                p0 = ex2_approx(p0);
                p1 = ex2_approx(p1);
                l2[u & 1] = f2_add(l2[u & 1], f2_pack(p0, p1));
                w8[u] = pack_bf16(p0, p1);
              }
              tc_st8(tS + (uint32_t)(half * 32 + e / 2), w8);
            }
          }
          float a0, a1;
          f2_unpack(f2_add(l2[0], l2[1]), a0, a1);
          l_run += a0 + a1;
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        mbar_arrive(p_bar(i));
      }
      // ---- the segment's result ----
      if (!dead) dead = __any_sync(0xffffffffu, !mbar_wait(o_bar(i), (c - 1u) & 1u, abort_flag));
      tc_fence_after();
      __threadfence_block();
      if (__any_sync(0xffffffffu, *odd_flag != 0 && !dead)) pt_add_odd<DH>(P, W.b, W.h, (long long)W.t0 * PT_KB, (long long)(W.t0 + W.nb) * PT_KB, len, keys, word, tO);
      const float inv = dead ? __int_as_float(0x7fffffff) : l_run == 0.f ? 0.f : 1.f / l_run;
      const size_t piece_at = (size_t)blockIdx.x * 2 + (W.x0 > W.x_begin ? 1 : 0), prow = piece_at * PT_ROWS + i * 128 + row;
      const bool none = l_run == 0.f && !dead;                       // the row sees nothing
#pragma unroll 1
      for (int d = 0; d < DH; d += 16) {
        float o[16];
        if (!dead) {
          tc_ld16(tO + (uint32_t)d, o);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = 0.f;
        }
        if (W.whole) {                       // staged over this thread's own query row, whose last scores have been formed
          uint32_t w8[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) w8[u] = none ? 0u : pack_bf16(o[2 * u] * inv, o[2 * u + 1] * inv);
          uint8_t* q = bp + i * C::QTILE;
          *reinterpret_cast<uint4*>(q + pt_q_off(row, d / 8)) = make_uint4(w8[0], w8[1], w8[2], w8[3]);
          *reinterpret_cast<uint4*>(q + pt_q_off(row, d / 8 + 1)) = make_uint4(w8[4], w8[5], w8[6], w8[7]);
        } else {                             // columns outside, rows inside: neighbouring threads write neighbouring 16 bytes
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(P.part_o + ((piece_at * (DH / 4) + (d + e) / 4) * PT_ROWS + i * 128 + row) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      if (W.whole) {                         // coalesced, as the queries came
        const long long off = valid ? (((long long)W.b * P.n + qi) * P.hq + W.h * P.group + hd) * DH : -1ll;
        __syncwarp();
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
          const long long o = __shfl_sync(0xffffffffu, off, u * RPI + lane / PIECES);
          if (o >= 0)
            *reinterpret_cast<uint4*>((bf16*)P.out + o + piece * 8) =
                *reinterpret_cast<const uint4*>(bp + i * C::QTILE + pt_q_off(quad * 32 + u * RPI + lane / PIECES, piece));
        }
        __syncwarp();
      }
      if (!W.whole && valid) {
        P.part_ml[prow * 2] = m_ref;
        P.part_ml[prow * 2 + 1] = dead ? __int_as_float(0x7fffffff) : l_run;
      }
      tc_fence_before();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace moa
