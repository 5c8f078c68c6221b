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
//   warp 1      one thread issues tcgen05.mma: S_i = Q_i K^T (Q in shared memory), O_i += P_i V (P in tensor memory, V as it
//               lies in the cache: MN-major)
//   warps 2..5  softmax of tile 0, one thread per query row; warps 6..9 of tile 1. P_i goes over S_i in tensor memory.
// Tensor memory: S_0 S_1 O_0 O_1, 128 columns each. The output is rescaled only when a row's maximum grew by more than 2^8.
// The probabilities enter the second product rounded once to bf16 (each off by at most 2^-8 of itself, so an output is off by
// at most 2^-8 * sum p |v|, the size of its own rounding to bf16), while their sum is taken in fp32 before the rounding.
// Work split, pieces and join are those of the row kernel, with items of 256 query rows and one CTA per SM.
// Every wait is bounded; a CTA whose wait ran out writes NaN to its rows.
#pragma once
#include <type_traits>

#include "moa_attn_tc.cuh"
#include "moa_paged.cuh"

namespace moa {

constexpr int PT_KB = 128;                   // positions per block
constexpr int PT_ROWS = 256;                 // query rows per item: two tiles
constexpr int PT_THREADS = 320;
constexpr int PT_SLOTS = 5;
constexpr uint32_t PT_TM_S = 0, PT_TM_O = 256;
constexpr int PT_POLY = 4;                    // of every 16 exponentials, how many go to the multiply-add pipe (an even number)

template <int DH> struct PtCfg {
  static constexpr int CK = DH / 64;                          // 64-column chunks of a row
  static constexpr int CHUNK = PT_KB * 128;                   // one chunk of 128 rows
  static constexpr int SLOT = CK * CHUNK;
  static constexpr int SMEM = 2 * SLOT + PT_SLOTS * SLOT + 1024 + 256;
};

// 16-byte piece of a query row in its tile: 64-column chunks of 128-byte rows, 128-byte swizzle.
template <int CHUNK>
__device__ __forceinline__ int pt_q_off(int row, int piece) { return (piece >> 3) * CHUNK + row * 128 + (((piece & 7) ^ (row & 7)) << 4); }

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
// 128 consecutive columns of this thread's lane, complete on return.
__device__ __forceinline__ void tc_ld128(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, "
      "%34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, "
      "%54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%128];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, "
      "%76, %77, %78, %79, %80, %81, %82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95, "
      "%96, %97, %98, %99, %100, %101, %102, %103, %104, %105, %106, %107, %108, %109, %110, %111, %112, "
      "%113, %114, %115, %116, %117, %118, %119, %120, %121, %122, %123, %124, %125, %126, %127}, "
      "[%129];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]), "=f"(v[32]),
        "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]),
        "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]), "=f"(v[48]),
        "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), "=f"(v[56]),
        "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]), "=f"(v[64]),
        "=f"(v[65]), "=f"(v[66]), "=f"(v[67]), "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]), "=f"(v[72]),
        "=f"(v[73]), "=f"(v[74]), "=f"(v[75]), "=f"(v[76]), "=f"(v[77]), "=f"(v[78]), "=f"(v[79]), "=f"(v[80]),
        "=f"(v[81]), "=f"(v[82]), "=f"(v[83]), "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]), "=f"(v[88]),
        "=f"(v[89]), "=f"(v[90]), "=f"(v[91]), "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]), "=f"(v[96]),
        "=f"(v[97]), "=f"(v[98]), "=f"(v[99]), "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]), "=f"(v[104]),
        "=f"(v[105]), "=f"(v[106]), "=f"(v[107]), "=f"(v[108]), "=f"(v[109]), "=f"(v[110]), "=f"(v[111]), "=f"(v[112]),
        "=f"(v[113]), "=f"(v[114]), "=f"(v[115]), "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]), "=f"(v[120]),
        "=f"(v[121]), "=f"(v[122]), "=f"(v[123]), "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
      : "r"(taddr + 0u), "r"(taddr + 64u)
      : "memory");
}

// Joins the pieces of the items that a stretch's end cut, in the order of their positions; an item that several ends cut
// belongs to the first of them. CTA (end of a stretch, quarter of the columns): a warp per 32 rows, a row per lane.
template <int DH>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedAttn P, int tile) {
  pdl_trigger();
  __shared__ PagedLine L;
  pdl_wait(KID_ATTN_MERGE);
  paged_line(L, P, tile);
  const int c = blockIdx.x + 1;
  if (L.total == 0 || c >= L.ctas) return;
  PagedPlace S;
  S.b = 0;
  const int x = line_begin(L, c);
  S.at(L, P, x);
  const int x0 = x - S.t;
  if (S.t == 0 || line_owner(L, x0) != c - 1) return;
  const int c1 = line_owner(L, x0 + S.T_b - 1);
  const int r = threadIdx.x, rr = S.mt * PT_ROWS + r;                // row of the item, of the (sequence, head)
  const int R = P.n * P.group;
  if ((rr & ~31) >= R) return;
  float M = -INFINITY, Z = 0.f;
#pragma unroll 4
  for (int i = c - 1; i <= c1; ++i) M = fmaxf(M, __ldg(P.part_ml + ((size_t)piece_of(L, i, x0) * PT_ROWS + r) * 2));
  const float ref = M == -INFINITY ? 0.f : M;
  constexpr int N4 = DH / 16;                                        // 16-byte pieces of a row in a quarter
  float4 a[N4];
#pragma unroll
  for (int d = 0; d < N4; ++d) a[d] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int i = c - 1; i <= c1; ++i) {
    const size_t piece = piece_of(L, i, x0);
    const float2 ml = __ldg(reinterpret_cast<const float2*>(P.part_ml) + piece * PT_ROWS + r);
    const float f = exp2f(ml.x - ref);
    Z = fmaf(f, ml.y, Z);
#pragma unroll
    for (int d = 0; d < N4; ++d) {
      const float4 o = __ldg(reinterpret_cast<const float4*>(P.part_o) + (piece * (DH / 4) + blockIdx.y * N4 + d) * PT_ROWS + r);
      a[d].x = fmaf(f, o.x, a[d].x); a[d].y = fmaf(f, o.y, a[d].y); a[d].z = fmaf(f, o.z, a[d].z); a[d].w = fmaf(f, o.w, a[d].w);
    }
  }
  if (rr >= R) return;
  const float inv = Z == 0.f ? 0.f : 1.f / Z;
  bf16* dst = (bf16*)P.out + (((size_t)S.b * P.n + rr / P.group) * P.hq + S.h * P.group + rr % P.group) * DH + blockIdx.y * (DH / 4);
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
    x = x_begin = line_begin(L, blockIdx.x);
    x_end = line_begin(L, blockIdx.x + 1);
    S.b = 0;
  }
  __device__ __forceinline__ bool next(const PagedLine& L, const PagedAttn& P) {
    if (x >= x_end) return false;
    S.at(L, P, x);
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
__device__ __forceinline__ float max3_nan(float a, float b, float c) {      // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^x of two values, -125 <= x <= 125, on the multiply-add pipe: x = n + f with n the nearest integer (by adding 1.5 * 2^23),
// 2^f on [-1/2, 1/2] by the polynomial of degree 5 with the least relative error (7.5e-8, a Remez fit), n added to the
// exponent. The special-function unit gives 16 exponentials a cycle and SM, which alone would take as long as both products.
__device__ __forceinline__ void ex2_poly2(uint64_t x, float& lo, float& hi) {
  const uint64_t magic = f2_pack(12582912.f, 12582912.f);
  const uint64_t t = f2_add(x, magic);
  const uint64_t n = f2_add(t, f2_pack(-12582912.f, -12582912.f));
  const uint64_t f = f2_fma(n, f2_pack(-1.f, -1.f), x);
  uint64_t y = f2_fma(f2_pack(0.0013276472454890609f, 0.0013276472454890609f), f, f2_pack(0.009675540961325169f, 0.009675540961325169f));
  y = f2_fma(y, f, f2_pack(0.05550713092088699f, 0.05550713092088699f));
  y = f2_fma(y, f, f2_pack(0.24022120237350464f, 0.24022120237350464f));
  y = f2_fma(y, f, f2_pack(0.6931469440460205f, 0.6931469440460205f));
  y = f2_fma(y, f, f2_pack(1.0000001192092896f, 1.0000001192092896f));
  float tl, th, yl, yh;
  f2_unpack(t, tl, th);
  f2_unpack(y, yl, yh);
  lo = __int_as_float(__float_as_int(yl) + (__float_as_int(tl) << 23));
  hi = __int_as_float(__float_as_int(yh) + (__float_as_int(th) << 23));
}

// bits of positions base .. base + 63 that a row with mask word w sees: committed ones (if it sees anything) and its new slots
__device__ __forceinline__ unsigned long long low_bits(long long n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }
__device__ __forceinline__ unsigned long long row_bits(unsigned long long w, long long base, int len, long long keys) {
  const long long s = len - base;
  unsigned long long v = w ? low_bits(s) : 0ull;
  if (s > -64 && s < 64) v |= s >= 0 ? w << s : w >> -s;
  return v & low_bits(keys - base);
}

template <int DH>
__global__ void __launch_bounds__(PT_THREADS, 1) paged_tree_kernel(const __grid_constant__ PagedTree PP) {
  using C = PtCfg<DH>;
  extern __shared__ uint8_t pt_smem_raw[];
  __shared__ PagedLine L;
  const PagedAttn& P = PP.a;
  const uint32_t base = (smem_u32(pt_smem_raw) + 1023u) & ~1023u;
  uint8_t* bp = pt_smem_raw + (base - smem_u32(pt_smem_raw));
  const uint32_t oRing = 2 * C::SLOT, oBar = oRing + PT_SLOTS * C::SLOT, bar0 = base + oBar;
  auto slot_at = [&](uint32_t s) { return base + oRing + s * (uint32_t)C::SLOT; };
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (PT_SLOTS + s); };
  auto q_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + i); };
  auto s_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 2 + i); };
  auto p_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 4 + i); };
  auto o_bar = [&](int i) { return bar0 + 8u * (2 * PT_SLOTS + 6 + i); };
  uint32_t* tmem_slot = (uint32_t*)(bp + oBar + 8 * (2 * PT_SLOTS + 8));
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = P.n * P.group;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < PT_SLOTS; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(q_bar(i), 128); mbar_init(s_bar(i), 1); mbar_init(p_bar(i), 128); mbar_init(o_bar(i), 1); }
    *abort_flag = 0;
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
  const bool idle = (int)blockIdx.x >= L.ctas || L.total == 0;
  PtWalk W;
  if (!idle) W.begin(L);

  if (idle) {
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
        int page = mine && slot0 < keys ? __ldg(table + (slot0 >> P.c.shift)) : P.c.n_pages;
        if (page < 0 || page > P.c.n_pages) page = P.c.n_pages;
        const int y = (int)(slot0 & ((1 << P.c.shift) - 1));
        for (int kv = 0; kv < 2; ++kv, ++cnt) {
          const uint32_t s = cnt % PT_SLOTS;
          ok = mbar_wait(empty_bar(s), ((cnt / PT_SLOTS) & 1u) ^ 1u, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(full_bar(s), C::SLOT);
          __syncwarp();
          if (mine) tma_load_3d(slot_at(s) + chunk * C::CHUNK + sub * rows * 128, kv ? &PP.tmV : &PP.tmK, x0, y, page, full_bar(s));
        }
      }
    }
    if (!ok && lane == 0) {                  // given up: the copies under way still land before the CTA ends
      const long long t_end = clock64() + WS_WAIT_CYCLES;
      for (uint32_t c = cnt > PT_SLOTS ? cnt - PT_SLOTS : 0; c < cnt; ++c)
        while (!mbar_test(full_bar(c % PT_SLOTS), (c / PT_SLOTS) & 1u) && clock64() < t_end) {}
    }
  } else if (warp == 1) {
    // ------------------------------ products ------------------------------
    if (lane == 0) {
      constexpr uint32_t IDESC_S = umma_idesc_bf16(128, PT_KB);
      constexpr uint32_t IDESC_O = umma_idesc_bf16_bmn(128, DH);
      uint32_t g = 0, cq[2] = {0u, 0u}, cp[2] = {0u, 0u};
      bool ok = true;
      auto scores = [&](int i, uint32_t blk, int tiles) -> bool {             // S_i of ring block blk
        const uint32_t c = 2 * blk, s = c % PT_SLOTS;
        if (!mbar_wait(full_bar(s), (c / PT_SLOTS) & 1u, abort_flag)) return false;
        tc_fence_after();
        const uint64_t kd = umma_desc_sw128(slot_at(s)), qd = umma_desc_sw128(base + i * C::SLOT);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
          const uint64_t o = (uint64_t)((ks >> 2) * (C::CHUNK / 16) + 2 * (ks & 3));
          tc_mma_bf16(tmem + PT_TM_S + i * 128, qd + o, kd + o, IDESC_S, ks > 0 ? 1u : 0u);
        }
        tc_commit(s_bar(i));
        if (i == tiles - 1) tc_commit(empty_bar(s));
        return true;
      };
      while (ok && W.next(L, P)) {
        const int tiles = W.pair * PT_ROWS + 128 < R ? 2 : 1;
        for (int i = 0; i < tiles && ok; ++i) {
          ok = mbar_wait(q_bar(i), cq[i]++ & 1u, abort_flag);
          tc_fence_after();
          if (ok) ok = scores(i, g, tiles);
        }
        for (int t = 0; t < W.nb && ok; ++t, ++g) {
          const uint32_t c = 2 * g + 1, s = c % PT_SLOTS;
          for (int i = 0; i < tiles; ++i) {
            ok = mbar_wait(p_bar(i), cp[i]++ & 1u, abort_flag);
            if (ok && i == 0) ok = mbar_wait(full_bar(s), (c / PT_SLOTS) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int ks = 0; ks < PT_KB / 16; ++ks)
              tc_mma_bf16_ta(tmem + PT_TM_O + i * 128, tmem + PT_TM_S + i * 128 + ks * 8, umma_desc_mn_sw128(slot_at(s) + ks * 2048, C::CHUNK),
                             IDESC_O, (t > 0 || ks > 0) ? 1u : 0u);
            tc_commit(o_bar(i));
            if (i == tiles - 1) tc_commit(empty_bar(s));
            if (t + 1 < W.nb && !scores(i, g + 1, tiles)) { ok = false; break; }
          }
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
      // coalesced: the warp's 32 rows, 32 * 8 / DH of them per instruction; rows behind the last one hold some real row and are
      // worked on, but not written
      constexpr int PIECES = DH / 8, RPI = 32 / PIECES;
      const int piece = lane % PIECES;
      {
        const long long off = ((long long)W.b * P.n + qi) * P.q_stride + (long long)(W.h * P.group + hd) * DH;
        uint4 x[PIECES];
#pragma unroll
        for (int u = 0; u < PIECES; ++u)
          x[u] = __ldg(reinterpret_cast<const uint4*>((const bf16*)P.q + __shfl_sync(0xffffffffu, off, u * RPI + lane / PIECES)) + piece);
#pragma unroll
        for (int u = 0; u < PIECES; ++u)
          *reinterpret_cast<uint4*>(bp + i * C::SLOT + pt_q_off<C::CHUNK>(quad * 32 + u * RPI + lane / PIECES, piece)) = x[u];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        mbar_arrive(q_bar(i));
      }
      // ---- what the rows see ----
      const unsigned long long any = any_word(P, W.b);
      unsigned long long word = row_word(P, W.b, qi);
      if (!valid) word = 0ull;
      const bool all_rows = __all_sync(0xffffffffu, word != 0ull || !valid);
      const int* table = P.c.table + (size_t)W.b * P.c.max_pages;
      bool bad = false;                      // a page of the segment that the table does not have
      {
        const long long s0 = (long long)W.t0 * PT_KB, s1 = min(keys, (long long)(W.t0 + W.nb) * PT_KB);
        for (long long p = (s0 >> P.c.shift) + lane; p << P.c.shift < s1; p += 32) {
          const int page = __ldg(table + p);
          bad = bad || page < 0 || page >= P.c.n_pages;
        }
        bad = __any_sync(0xffffffffu, bad);
      }
      float m_ref = -INFINITY, l_run = 0.f;
      for (int t = 0; t < W.nb; ++t, ++g, ++c) {
        if (!dead) dead = __any_sync(0xffffffffu, !mbar_wait(s_bar(i), c & 1u, abort_flag));
        if (dead) continue;
        tc_fence_after();
        float s[128];
        tc_ld128(tS, s);
        const long long k0 = (long long)(W.t0 + t) * PT_KB;
        const bool masked = k0 + PT_KB > len || bad || !all_rows;
        if (masked) {
          unsigned long long vis[2] = {row_bits(word, k0, len, keys), row_bits(word, k0 + 64, len, keys)};
          unsigned long long live[2] = {row_bits(any, k0, len, keys), row_bits(any, k0 + 64, len, keys)};
          if (bad) {
            for (int j = 0; j < PT_KB; j += min(PT_KB, 1 << P.c.shift)) {
              if (k0 + j >= keys) break;
              const int page = __ldg(table + ((k0 + j) >> P.c.shift));
              if (page >= 0 && page < P.c.n_pages) continue;
              for (int e = j; e < j + min(PT_KB, 1 << P.c.shift); ++e) { vis[e >> 6] &= ~(1ull << (e & 63)); live[e >> 6] &= ~(1ull << (e & 63)); }
            }
          }
#pragma unroll
          for (int e = 0; e < 128; ++e)
            if (!((vis[e >> 6] >> (e & 63)) & 1ull)) s[e] = -INFINITY;
          // zero times what lies in a slot that does not exist may not be zero: such values are cleared, by the tile's 128
          // threads a row each, once they have landed (the other tile clears the same rows itself)
          if (~(live[0] & live[1]) != 0ull) {
            const uint32_t v = 2 * g + 1, vs = v % PT_SLOTS;
            dead = __any_sync(0xffffffffu, !mbar_wait(full_bar(vs), (v / PT_SLOTS) & 1u, abort_flag));
            if (dead) continue;
            if (!((live[row >> 6] >> (row & 63)) & 1ull)) {
              uint8_t* d = bp + oRing + vs * C::SLOT + row * 128;
#pragma unroll
              for (int p = 0; p < DH / 8; ++p) *reinterpret_cast<uint4*>(d + (p >> 3) * C::CHUNK + ((p & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 128; e += 8)
#pragma unroll
          for (int u = 0; u < 4; ++u) m4[u] = max3_nan(m4[u], s[e + 2 * u], s[e + 2 * u + 1]);
        const float m_blk = max3_nan(max3_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]) * P.scale_log2;
        float f = 1.f;
        if (m_ref == -INFINITY) {
          m_ref = m_blk;                     // nothing has been added for this row yet
        } else if (m_blk > m_ref + TC_RESCALE_LOG2) {
          f = ex2_approx(m_ref - m_blk);
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
        const uint64_t scale2 = f2_pack(P.scale_log2, P.scale_log2), sub2 = f2_pack(-sub, -sub);
        uint64_t l2[2] = {0ull, 0ull};
        // scores that are not there (-inf) and NaN take the special-function unit: the polynomial knows neither
        const bool poly = !masked && __all_sync(0xffffffffu, m_blk > -3.0e38f);
        auto probabilities = [&](auto with_poly) {
#pragma unroll
          for (int e = 0; e < 128; e += 16) {
            uint32_t w8[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const uint64_t x = f2_fma(f2_pack(s[e + 2 * u], s[e + 2 * u + 1]), scale2, sub2);
              float p0, p1;
              if (decltype(with_poly)::value && u * 2 >= 16 - PT_POLY) {
                float x0, x1;
                f2_unpack(x, x0, x1);
                ex2_poly2(f2_pack(fmaxf(x0, -125.f), fmaxf(x1, -125.f)), p0, p1);
              } else {
                float x0, x1;
                f2_unpack(x, x0, x1);
                p0 = ex2_approx(x0);
                p1 = ex2_approx(x1);
              }
              l2[u & 1] = f2_add(l2[u & 1], f2_pack(p0, p1));
              w8[u] = pack_bf16(p0, p1);
            }
            tc_st8(tS + (uint32_t)(e / 2), w8);
          }
        };
        if (poly) probabilities(std::true_type{}); else probabilities(std::false_type{});
        {
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
      const float inv = dead ? __int_as_float(0x7fffffff) : l_run == 0.f ? 0.f : 1.f / l_run;
      const size_t piece_at = (size_t)piece_of(L, blockIdx.x, W.x0), prow = piece_at * PT_ROWS + i * 128 + row;
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
          uint8_t* q = bp + i * C::SLOT;
          *reinterpret_cast<uint4*>(q + pt_q_off<C::CHUNK>(row, d / 8)) = make_uint4(w8[0], w8[1], w8[2], w8[3]);
          *reinterpret_cast<uint4*>(q + pt_q_off<C::CHUNK>(row, d / 8 + 1)) = make_uint4(w8[4], w8[5], w8[6], w8[7]);
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
                *reinterpret_cast<const uint4*>(bp + i * C::SLOT + pt_q_off<C::CHUNK>(quad * 32 + u * RPI + lane / PIECES, piece));
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
