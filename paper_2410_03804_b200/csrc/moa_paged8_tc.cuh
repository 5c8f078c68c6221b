// Attention of many query rows per key / value head over an 8-bit paged cache, on the 5th-generation tensor cores (sm_100a): the rows
// of a kept draft tree (up to 64 rows x the heads of a group).
//
// The products, the softmax and the work split are those of moa_paged_tc.cuh: items of 256 query rows in two tiles of 128 that take
// turns over a stream of blocks of 128 positions, one CTA per SM, S_i = Q_i K^T and O_i += P_i V with P_i over S_i in tensor memory.
// What differs is where the operands come from, and that all of them are fp16:
//   warps 0..3, 4..7  softmax of tile 0 and of tile 1, a thread per query row
//   warp 8            tcgen05.mma
//   warp 9            what the softmax has to know of a block's scales
//   warps 10..12, 13..15  make the operands, the keys and the values, two blocks of each in shared memory: the records' codes go through
//                     registers, a block ahead, and become fp16, exactly, in the order that the products read (128-byte swizzle; the
//                     values transposed, as their records hold them, so both operands are K-major)
// Open slots come from the 16-bit ring; a kernel before this one (paged8_open_kernel) scales them into fp16's range by a power of two
// per 16 positions, in the operands' order.
// A scale belongs to 16 positions, which are 16 neighbouring scores of a row: the keys' scale is a factor of the exponent's
// multiply-add, and of the maximum of the 16 scores; the values' scale, relative to a power of two above all that the item has met,
// is a term of its addend, 2^(x + log2 r) = r 2^x, and is divided out of the 16 probabilities' sum again.
// The probabilities are rounded once to fp16 (2^-11 of themselves), a quarter of the outputs' own rounding to bf16.
// A tile's first 64 probabilities are handed over while the other 64 are made, so half of their product is done when those come.
// Measured: 16 sequences x 61 rows x 64 heads over 4090 positions: 208 us, with the commit 216 (the row kernel: 1466); 61 rows x 32
// heads over 2045: 31.7 and 36.4. What it took to get there, us of the large case: the masks out of the softmax's loop (380 to 350),
// operands' addresses that are constants apart, their registers not live across a call, and the open slots' work in a kernel of its
// own (here it ran cold, once per item, for 100000 cycles; together to 263), loops in place of unrolled halves (to 212: a quarter of
// the instruction cache's requests had missed, 8 % do now), probabilities in two halves (to 208).
// Every wait is bounded; a CTA whose wait ran out writes NaN to its rows (the serving calls have no status word).
#pragma once
#include "moa_paged8.cuh"
#include "moa_paged_tc.cuh"

namespace moa {

constexpr int P8T_THREADS = 512;
constexpr int P8T_AT = 32;                   // scores that the softmax's loops take at a time
constexpr int P8T_TABLE_WARP = 9, P8T_CONV_WARP = 10;

struct P8Table {                             // of one block of 128 positions: per 16 of them
  float ks[8];                               // scale of the keys
  float lr[8];                               // log2 of the values' scale in units of vref, + P8_BIAS
  float ir[8];                               // and its inverse
  uint32_t live[4];                          // bit per position: whether there is a row
  float fv, vref;                            // factor that takes sums from the last block's vref to this one's
  float pad[2];
};

template <int DH> struct P8tCfg {
  static constexpr int QTILE = 128 * DH * 2, KTILE = PT_KB * DH * 2;
  static constexpr int QCHUNK = 128 * 128, KCHUNK = PT_KB * 128, VCHUNK = DH * 128;          // 64 columns: of queries, of keys; 64 positions of values
  static constexpr int REC = P8Cfg<DH>::REC;
  static constexpr int O_K = 2 * QTILE, O_V = O_K + 2 * KTILE, O_TAB = O_V + 2 * KTILE;          // two of keys, two of values
  static constexpr int O_BAR = O_TAB + 4 * (int)sizeof(P8Table);
  static constexpr int SMEM = O_BAR + 256 + 1024;
};

__host__ __device__ constexpr uint32_t umma_idesc_f16(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// 32 consecutive columns of this thread's lane in one instruction
__device__ __forceinline__ void tc_ld32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// Four codes (plus 128) of a word as fp16, in order.
__device__ __forceinline__ uint2 p8_codes_in_order(uint32_t w) {
  return make_uint2(p8_less_bias(__byte_perm(w, 0x64646464u, 0x4140)), p8_less_bias(__byte_perm(w, 0x64646464u, 0x4342)));
}
// Barrier over three converting warps that also ORs a flag: who gives up takes all of them along.
template <int ID>
__device__ __forceinline__ bool p8t_bar_any(bool mine) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred.aligned q, %2, 96, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(mine ? 1u : 0u), "n"(ID)
      : "memory");
  return r != 0u;
}
// Power of two that brings values of at most m to [2^t, 2^(t+1)), and its inverse; 1 where there is none.
__device__ __forceinline__ void p8_range_to(float m, int t, float& up, float& down) {
  const int e = (int)(__float_as_uint(m) >> 23);
  const bool fit = e > t + 1 && e < 255;
  up = fit ? __uint_as_float((uint32_t)(254 + t - e) << 23) : 1.f;
  down = fit ? __uint_as_float((uint32_t)(e - t) << 23) : 1.f;
}
__device__ __forceinline__ float warp_top(uint32_t top) { return __uint_as_float(__reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16)) << 16); }

// One unit of work of a converting warp: 16 positions of keys, or of values.
template <int DH>
struct P8Convert {
  using C = P8tCfg<DH>;
  static constexpr int UNITS = DH / 32;      // a closed block's keys, or values, are so many units: 16 bytes of codes per lane
  // Where a lane's 16 bytes of unit r lie in a record. The lanes are dealt out so that the stores to the operand, rows of 128 bytes
  // whose 16-byte pieces are swizzled by the row, do not meet in a bank.
  static __device__ __forceinline__ int at_keys(int r) {
    const int lane = threadIdx.x & 31, x = (lane >> 2) & 1;
    return ((x ^ (r & 1)) * (DH / 64) + (r >> 1)) * 512 + ((lane >> 3) * 2 + x) * 64 + (lane & 3) * 16;
  }
  // Where they go: rows j * 16 + row of the keys; p: r & 1. Blocks lie 16 rows, 2048 bytes, apart.
  static __device__ __forceinline__ uint32_t to_keys(int p, int e) {
    const int lane = threadIdx.x & 31, tq = lane & 3, x = (lane >> 2) & 1, row = 2 * ((lane >> 3) * 2 + x) + (x ^ p);
    return (uint32_t)(row * 128 + (((2 * tq + e) ^ (row & 7)) << 4));
  }
  static __device__ __forceinline__ void store_keys(uint8_t* K, uint32_t to0, uint32_t to1, const uint4& c) {
    const uint2 a = p8_codes_in_order(c.x), b = p8_codes_in_order(c.y), d = p8_codes_in_order(c.z), e = p8_codes_in_order(c.w);
    *reinterpret_cast<uint4*>(K + to0) = make_uint4(a.x, a.y, b.x, b.y);
    *reinterpret_cast<uint4*>(K + to1) = make_uint4(d.x, d.y, e.x, e.y);
  }
  // dim % 8 of a lane's values
  static __device__ __forceinline__ int value_row() {
    const int lane = threadIdx.x & 31, i = (lane >> 2) & 3;
    return (i >> 1) * 4 + (lane >> 4 ? 1 + (i & 1) : 3 * (i & 1));
  }
  static __device__ __forceinline__ int at_values(int k) { return P8Cfg<DH>::CODES + k * 512 + value_row() * 64 + (threadIdx.x & 3) * 16; }
  // where four tokens of a dim, 8 bytes, go in the transposed values
  static __device__ __forceinline__ uint32_t to_values(int j) {
    const int row = value_row(), tq = threadIdx.x & 3;
    return (uint32_t)((j >> 2) * C::VCHUNK + row * 128 + (((2 * (j & 3) + (tq >> 1)) ^ row) << 4) + (tq & 1) * 8);
  }
  static __device__ __forceinline__ void store_values(uint8_t* V, uint32_t to, int k, const uint4& c) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint2*>(V + to + (32 * k + 8 * i) * 128) = p8_codes_in_order(w[i]);
  }
  // all units of closed block j
  template <bool VALUES>
  static __device__ __forceinline__ void load(uint4* c, const uint8_t* rec) {
#pragma unroll
    for (int r = 0; r < UNITS; ++r) c[r] = __ldcg(reinterpret_cast<const uint4*>(rec + (VALUES ? at_values(r) : at_keys(r))));
  }
  template <bool VALUES>
  static __device__ __forceinline__ void store(uint8_t* to, int j, const uint4* c) {
#pragma unroll
    for (int r = 0; r < UNITS; ++r) {
      if (VALUES) store_values(to, to_values(j), r, c[r]);
      else store_keys(to + (r >> 1) * C::KCHUNK + j * 2048, to_keys(r & 1, 0), to_keys(r & 1, 1), c[r]);
    }
  }
  // block j from an open block's record
  template <bool VALUES>
  static __device__ __forceinline__ void copy(uint8_t* to, int j, const uint8_t* open) {
    uint4 c[DH / 16];
#pragma unroll
    for (int u = 0; u < DH / 16; ++u)
      c[u] = __ldcg(reinterpret_cast<const uint4*>(open + (VALUES ? 32 * DH : 0)) + u * 32 + (threadIdx.x & 31));
#pragma unroll
    for (int u = 0; u < DH / 16; ++u) {
      const int i = u * 32 + (threadIdx.x & 31);
      const int row = VALUES ? i >> 1 : j * 16 + i / (DH / 8), piece = VALUES ? 2 * (j & 3) + (i & 1) : i % (DH / 8);
      uint8_t* at = to + (VALUES ? (j >> 2) * C::VCHUNK : (piece >> 3) * C::KCHUNK) + row * 128;
      *reinterpret_cast<uint4*>(at + (((piece & 7) ^ (row & 7)) << 4)) = c[u];
    }
  }
};

// An open block of one head as the tree kernel wants it: keys fp16 [16][DH], values fp16 [DH][16], their scales, a bit per row that is
// there, and whether a value is not finite (such values are zeros here, and added to the rows that see them by themselves).
template <int DH> struct P8Open {
  static constexpr int BYTES = 64 * DH + 16, MAX = P8_RING / 16;
  static __device__ __forceinline__ uint8_t* at(uint8_t* open, const PagedView& c, int b, int h, int i) { return open + ((size_t)(b * c.hkv + h) * MAX + i) * BYTES; }
};
// Makes them, and takes the call's new rows to the ring: a CTA per block, a warp for the keys and one for the values. (Done where the
// tree kernel needs them, this code ran once per item, cold, at some 40000 cycles.)
template <int DH>
__global__ void __launch_bounds__(64) paged8_open_kernel(const Paged8 PP, uint8_t* open) {
  pdl_trigger();
  pdl_wait(KID_APPEND);
  const PagedAttn& P = PP.a;
  const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31;
  const bool values = threadIdx.x >= 32;
  const int cap = (int)P.c.cap(), len = min(P.c.len[b], cap);
  if (len < 0) return;
  const int keys = min(len + P.n_new, cap), s0 = ((len >> 4) + i) * 16;
  if (s0 >= keys) return;
  const unsigned long long any = any_word(P, b);
  const int slot = s0 + (lane & 15);
  const uint32_t live = __ballot_sync(0xffffffffu, slot < keys && (slot < len || ((any >> (slot - len)) & 1ull) != 0ull)) & 0xffffu;
  uint8_t* to = P8Open<DH>::at(open, P.c, b, h, i);
  bf16* const ring = (bf16*)(values ? P.c.v : P.c.k);
  const bf16* const fresh = (const bf16*)(values ? P.v_new : P.k_new);
  // 16 bytes of a row; a new one goes to the ring on the way
  auto get = [&](int t, int piece) -> uint4 {
    if (!((live >> t) & 1u)) return make_uint4(0u, 0u, 0u, 0u);
    uint4* at = reinterpret_cast<uint4*>(ring + p8_ring_row(P.c, b, s0 + t, h, DH)) + piece;
    if (s0 + t < len || !fresh) return __ldcg(at);
    const uint4 x = __ldcg(reinterpret_cast<const uint4*>(fresh + ((long long)b * P.n + (s0 + t - len)) * P.new_stride + (long long)h * DH) + piece);
    *at = x;
    return x;
  };
  uint32_t top = 0u;
  float up, scale;
  if (!values) {
    const int gq = lane >> 2, tq = lane & 3;
    uint4 x[2][DH / 64][2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < DH / 64; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[p][k][e] = get(2 * gq + p, k * 8 + tq * 2 + e);
          top = finite2_max(top, x[p][k][e]);
        }
    p8_range_to(warp_top(top), 14, up, scale);                       // (a key that is not finite stays one: its scores are the rows' own that see it)
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < DH / 64; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float f[8];
          bf16x8_to_float(x[p][k][e], f);
          reinterpret_cast<uint4*>(to + (2 * gq + p) * DH * 2)[k * 8 + tq * 2 + e] =
              make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up), pack_f16(f[6] * up, f[7] * up));
        }
    if (lane == 0) {
      *reinterpret_cast<float*>(to + 64 * DH) = scale;
      *reinterpret_cast<uint32_t*>(to + 64 * DH + 8) = live;
    }
  } else {
    const int tq = lane & 3, c = lane >> 2;
    uint4 x[DH / 64][4];
    bool odd = false;
#pragma unroll
    for (int u = 0; u < DH / 64; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        x[u][t] = get(4 * tq + t, u * 8 + c);
        odd = odd || odd_any(x[u][t]);
        x[u][t] = odd_cleared(x[u][t]);
        top = finite2_max(top, x[u][t]);
      }
    odd = __any_sync(0xffffffffu, odd);
    const float m = warp_top(top);
    p8_range_to(m, 6, up, scale);
    if (m < 0x1p-100f) up = scale = 0.f;     // zeros, or held as them
#pragma unroll
    for (int u = 0; u < DH / 64; ++u) {
      float f[4][8];
#pragma unroll
      for (int t = 0; t < 4; ++t) bf16x8_to_float(x[u][t], f[t]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<uint2*>(to + 32 * DH + ((u * 8 + c) * 8 + e) * 32 + tq * 8) = make_uint2(pack_f16(f[0][e] * up, f[1][e] * up), pack_f16(f[2][e] * up, f[3][e] * up));
    }
    if (lane == 0) {
      *reinterpret_cast<float*>(to + 64 * DH + 4) = scale;
      *reinterpret_cast<uint32_t*>(to + 64 * DH + 12) = odd ? 1u : 0u;
    }
  }
}

// The operand of a block of 128 positions with blocks of 16 that are open, behind the end, or on pages that the table does not have. The
// latter two keep what was there: their scores are masked, and zero times a finite value is zero.
template <int DH, bool VALUES>
__device__ __noinline__ void p8t_ragged(const Paged8& PP, int b, int h, int blk0, const uint8_t* rec, int len, int keys, uint8_t* to, int cw) {
  using X = P8Convert<DH>;
  const PagedAttn& P = PP.a;
#pragma unroll 1
  for (int j = cw; j < 8; j += 3) {
    const int blk = blk0 + j, i = blk - (len >> 4);
    const uint8_t* from = (const uint8_t*)__shfl_sync(0xffffffffu, (unsigned long long)rec, j);
    if (from) {
      uint4 c[X::UNITS];
      X::template load<VALUES>(c, from);
      X::template store<VALUES>(to, j, c);
    } else if (i >= 0 && blk * 16 < keys) {
      X::template copy<VALUES>(to, j, P8Open<DH>::at(PP.open, P.c, b, h, i));
    }
  }
}

// Scores of positions that a row does not see become -inf, in tensor memory, 16 at a time, before the softmax looks at them (the last
// block of an item, as a rule). With the masks in the softmax's loop its instructions were half as many again, all of them on the
// pipe that the maxima, roundings and code bytes need too. True where 16 scores' factor is zero, so that -inf times it is none.
__device__ __noinline__ bool p8t_mask(uint32_t tS, const P8Table* tab, unsigned long long vis0, unsigned long long vis1, float factor) {
  bool zero = false;
#pragma unroll 1
  for (int b = 0; b < 8; ++b) {
    const uint32_t v = (uint32_t)((b < 4 ? vis0 : vis1) >> (16 * (b & 3))) & 0xffffu;
    if (!__any_sync(0xffffffffu, v != 0xffffu)) continue;
    float s[16];
    tc_ld16(tS + (uint32_t)(16 * b), s);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = (v >> e) & 1u ? s[e] : -INFINITY;
    tc_st16(tS + (uint32_t)(16 * b), s);
    zero = zero || !(tab->ks[b] * factor > 0.f);
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
  return zero;
}
// Probabilities over their scores for rows with scores far from zero, the differences taken before they are scaled; returns their sum.
__device__ __noinline__ float p8t_slow(uint32_t tS, const P8Table* tab, float down, float sub, float scale) {
  float l = 0.f;
#pragma unroll 1
  for (int b = 0; b < 8; ++b) {              // the probabilities, two to a column, stay behind the scores that are read
    float s[16], g = 0.f;
    tc_ld16(tS + (uint32_t)(16 * b), s);
    const float kd = tab->ks[b] * down, lr = tab->lr[b];
    uint32_t w8[8];
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p0 = s[e] == -INFINITY ? 0.f : ex2_approx(fmaf(__fmul_rn(s[e], kd) - sub, scale, lr));
      const float p1 = s[e + 1] == -INFINITY ? 0.f : ex2_approx(fmaf(__fmul_rn(s[e + 1], kd) - sub, scale, lr));
      g += p0 + p1;
      w8[e / 2] = pack_f16(p0, p1);
    }
    l = fmaf(g, tab->ir[b], l);
    tc_st8(tS + (uint32_t)(8 * b), w8);
  }
  return l;
}
// Adds to a row's output (tensor memory, at tO) the values that are not finite of the open slots that it sees among positions
// from .. to - 1. A whole warp; the rows' words may differ.
template <int DH>
__device__ __noinline__ void p8t_add_odd(const PagedAttn& P, int b, int h, long long from, long long to, int len, int keys, unsigned long long word, uint32_t tO) {
  for (int d = 0; d < DH; d += 16) {
    float o[16];
    tc_ld16(tO + (uint32_t)d, o);
    for (int key = len & ~15; key < keys; ++key) {
      const bool sees = key < len ? word != 0ull : ((word >> (key - len)) & 1ull) != 0ull;
      if (key < from || key >= to || !sees) continue;
      const bf16* v = (const bf16*)P.c.v + p8_ring_row(P.c, b, key, h, DH) + d;
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

// The blocks' keys, or values, as operands at `to` (two places), by three warps; full, empty: the places' barriers, 8 bytes apart. The
// next block's codes are under way, in registers, while this one's place is waited for and filled.
template <int DH, bool VALUES>
__device__ __forceinline__ void p8t_operands(const Paged8& PP, const PagedLine& L, uint8_t* to, uint32_t full, uint32_t empty, int cw,
                                             volatile int* abort_flag) {
  using X = P8Convert<DH>;
  const PagedAttn& P = PP.a;
  const int lane = threadIdx.x & 31, cap = (int)P.c.cap();
  PtWalk W;
  W.begin(L);
  uint32_t g = 0;
  while (W.next(L, P)) {
    const int len = min(L.len[W.b], cap), keys = min(len + P.n_new, cap), shut = len >> 4;
    uint4 c[3][X::UNITS];                    // blocks cw, cw + 3 and cw + 6 of 16 positions
    unsigned there = 0u;
    const uint8_t *rec = nullptr, *last = nullptr;                   // a record per lane, looked up a block ahead of its loads; the loaded block's
    if (lane < 8 && W.t0 * 8 + lane < shut) rec = p8_record<DH>(P.c, PP.pages, PP.page_bytes, W.b, W.h, W.t0 * 8 + lane);
#pragma unroll 1
    for (int t = -1; t < W.nb; ++t) {
      if (t >= 0) {
        uint8_t* const at = to + (g & 1u) * P8tCfg<DH>::KTILE;
        const bool good = __all_sync(0xffffffffu, mbar_wait(empty + 8u * (g & 1u), ((g >> 1) & 1u) ^ 1u, abort_flag));
        if (good) {
          if (there == 0xffu) {
#pragma unroll 1
            for (int j = cw; j < 8; j += 3) {
              X::template store<VALUES>(at, j, c[0]);
#pragma unroll
              for (int r = 0; r < X::UNITS; ++r) { c[0][r] = c[1][r]; c[1][r] = c[2][r]; }
            }
          } else {
            p8t_ragged<DH, VALUES>(PP, W.b, W.h, (W.t0 + t) * 8, last, len, keys, at, cw);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (p8t_bar_any<VALUES ? 3 : 2>(!good)) return;
        if (cw == 0 && lane == 0) mbar_arrive(full + 8u * (g & 1u));
        ++g;
      }
      there = __ballot_sync(0xffffffffu, rec != nullptr);
      last = rec;
      if (there == 0xffu) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const unsigned long long from = __shfl_sync(0xffffffffu, (unsigned long long)rec, (cw + 3 * i) & 7);          // (the third warp's ninth block is none)
          X::template load<VALUES>(c[i], (const uint8_t*)from);
        }
      } else {                               // (nothing stays in these registers across the call above)
#pragma unroll
        for (int i = 0; i < 3 * X::UNITS; ++i) c[i / X::UNITS][i % X::UNITS] = make_uint4(0u, 0u, 0u, 0u);
      }
      const int blk = (W.t0 + t + 2) * 8 + lane;
      rec = t + 2 < W.nb && lane < 8 && blk < shut ? p8_record<DH>(P.c, PP.pages, PP.page_bytes, W.b, W.h, blk) : nullptr;
    }
  }
}

template <int DH>
__global__ void __launch_bounds__(P8T_THREADS, 1) paged8_tree_kernel(const __grid_constant__ Paged8 PP) {
  using C = P8tCfg<DH>;
  extern __shared__ uint8_t pt_smem_raw[];
  __shared__ PagedLine L;
  const PagedAttn& P = PP.a;
  const uint32_t base = (smem_u32(pt_smem_raw) + 1023u) & ~1023u;
  uint8_t* bp = pt_smem_raw + (base - smem_u32(pt_smem_raw));
  const uint32_t bar0 = base + C::O_BAR;
  auto q_bar = [&](int i) { return bar0 + 8u * i; };
  auto s_bar = [&](int i) { return bar0 + 8u * (2 + i); };
  auto p_bar = [&](int i) { return bar0 + 8u * (4 + i); };
  auto o_bar = [&](int i) { return bar0 + 8u * (6 + i); };
  // operands of block blk: kv 0 keys, 1 values
  auto full_bar = [&](int kv, uint32_t blk) { return bar0 + 64u + 16u * kv + 8u * (blk & 1u); };
  auto empty_bar = [&](int kv, uint32_t blk) { return bar0 + 96u + 16u * kv + 8u * (blk & 1u); };
  auto table_bar = [&](uint32_t blk) { return bar0 + 128u + 8u * (blk & 3u); };
  auto h_bar = [&](int i) { return bar0 + 160u + 8u * i; };
  uint32_t* tmem_slot = (uint32_t*)(bp + C::O_BAR + 176);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  volatile int* odd_flag = abort_flag + 1;   // an open slot's value that is not finite was met
  P8Table* const tabs = (P8Table*)(bp + C::O_TAB);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = P.n * P.group, cap = (int)P.c.cap();
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_bar(i), 128);
      mbar_init(s_bar(i), 1);
      mbar_init(p_bar(i), 128);
      mbar_init(h_bar(i), 128);
      mbar_init(o_bar(i), 1);
    }
    for (uint32_t i = 0; i < 4; ++i) mbar_init(table_bar(i), 1);
    for (uint32_t i = 0; i < 4; ++i) { mbar_init(full_bar((int)(i >> 1), i), 1); mbar_init(empty_bar((int)(i >> 1), i), 1); }
    *abort_flag = *odd_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int i = threadIdx.x; i < 2 * C::KTILE / 16; i += P8T_THREADS) reinterpret_cast<uint4*>(bp + C::O_V)[i] = make_uint4(0u, 0u, 0u, 0u);      // (finite)
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  pdl_wait(KID_ATTN);
  paged_line(L, P, PT_KB);                   // ends with a barrier
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const bool idle = L.x_begin == L.x_end;

  if (warp >= 8) {
    if (idle) {
      if (threadIdx.x == 256) P.joins[blockIdx.x * 8] = 0;
    } else if (warp == P8T_TABLE_WARP) {
      // ------------------------------ scales ------------------------------
      if (lane == 0) {                       // the item that the end of this stretch cuts first, for the join
        PagedPlace S;
        S.at(L, P, L.x_end - 1);
        const int x0 = L.x_end - 1 - S.t;
        int4* j = reinterpret_cast<int4*>(P.joins) + blockIdx.x * 2;
        const bool cut = x0 >= L.x_begin && x0 + S.T_b > L.x_end;
        j[0] = make_int4(cut ? line_owner(L, x0 + S.T_b - 1) : 0, x0 > L.x_begin ? 1 : 0, S.b, S.h);
        j[1] = make_int4(S.mt, 0, 0, 0);
      }
      PtWalk W;
      W.begin(L);
      uint32_t g = 0;
      bool ok = true;
      while (ok && W.next(L, P)) {
        const int len = min(L.len[W.b], cap), keys = min(len + P.n_new, cap), shut = len >> 4;
        float vref = 0.f;
        for (int t = 0; t < W.nb; ++t, ++g) {
          const int blk0 = (W.t0 + t) * 8;
          const uint8_t* rec = lane < 8 && blk0 + lane < shut ? p8_record<DH>(P.c, PP.pages, PP.page_bytes, W.b, W.h, blk0 + lane) : nullptr;
          const float2 sc = rec ? __ldcg(reinterpret_cast<const float2*>(rec + 2 * P8Cfg<DH>::CODES)) : make_float2(0.f, 0.f);
          float ks = sc.x, vs = sc.y;
          uint32_t live = rec ? 0xffffu : 0u;
          if (lane < 8 && rec == nullptr) {
            ks = 1.f;                        // (zeros times it)
            if (blk0 + lane >= shut && (blk0 + lane) * 16 < keys) {
              const uint4 o = __ldcg(reinterpret_cast<const uint4*>(P8Open<DH>::at(PP.open, P.c, W.b, W.h, blk0 + lane - shut) + 64 * DH));
              ks = __uint_as_float(o.x);
              vs = __uint_as_float(o.y);
              live = o.z;
              if (o.w) *odd_flag = 1;
            }
          }
          const float most = __uint_as_float(__reduce_max_sync(0xffffffffu, vs >= 0.f ? __float_as_uint(vs) : 0u));       // NaN aside
          float fv = 1.f;
          if (most > vref) {                 // 4 to 8 times the largest, so that it is rarely passed
            const float ref = __uint_as_float(((__float_as_uint(most) >> 23) + 3u) << 23);
            fv = vref == 0.f ? 1.f : vref * __uint_as_float((254u << 23) - __float_as_uint(ref));
            vref = ref;
          }
          // Written over the table of four blocks before, whose probabilities had to be there before the scores of two blocks before
          // this one, which are complete. (Scores wait for the table, so this wait cannot fall a phase behind.)
          P8Table* tab = tabs + (g & 3u);
          ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(0, g), ((g >> 1) & 1u) ^ 1u, abort_flag));
          if (!ok) break;
          if (lane < 8) {
            // values that are zeros have any scale; one below 2^-60 of the largest counts as that (off by 2^-53 of the largest value)
            const float r = vs == 0.f ? 1.f : vs * __uint_as_float((254u << 23) - __float_as_uint(vref == 0.f ? 1.f : vref));
            const float q = r < 0x1p-60f ? 0x1p-60f : r;             // (a NaN stays one)
            tab->ks[lane] = ks;
            tab->lr[lane] = log2f(q) + P8_BIAS;
            tab->ir[lane] = 1.f / q;
            reinterpret_cast<uint16_t*>(tab->live)[lane] = (uint16_t)live;
          }
          if (lane == 0) {
            tab->fv = fv;
            tab->vref = vref == 0.f ? 1.f : vref;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(table_bar(g));
        }
      }
    } else if (warp >= P8T_CONV_WARP) {
      // ------------------------------ operands: three warps for the keys, three for the values ------------------------------
      if (warp < P8T_CONV_WARP + 3) p8t_operands<DH, false>(PP, L, bp + C::O_K, full_bar(0, 0), empty_bar(0, 0), warp - P8T_CONV_WARP, abort_flag);
      else p8t_operands<DH, true>(PP, L, bp + C::O_V, full_bar(1, 0), empty_bar(1, 0), warp - P8T_CONV_WARP - 3, abort_flag);
    } else if (warp == 8) {
      // ------------------------------ products ------------------------------
      // The whole warp walks the loops, so that addresses and descriptors stay in uniform registers; one elected lane issues.
      constexpr uint32_t IDESC_S = umma_idesc_f16(128, PT_KB), IDESC_O = umma_idesc_f16(128, DH);
      PtWalk W;
      W.begin(L);
      uint32_t g = 0, cq[2] = {0u, 0u}, c[2] = {0u, 0u};        // block of the segment's first block; queries, blocks of the tiles
      bool ok = true;
      const bool leader = pt_elect();
      auto scores = [&](int i, uint32_t blk, int tiles) -> bool {               // S_i of block blk
        if (!__all_sync(0xffffffffu, mbar_wait(full_bar(0, blk), (blk >> 1) & 1u, abort_flag) && mbar_wait(table_bar(blk), (blk >> 2) & 1u, abort_flag))) return false;
        tc_fence_after();
        const uint64_t qd = umma_desc_sw128(base + i * C::QTILE), kd = umma_desc_sw128(base + C::O_K + (blk & 1u) * C::KTILE);
        const uint32_t d = tmem + PT_TM_S + i * 128;
        if (leader) {
#pragma unroll
          for (int ks = 0; ks < DH / 16; ++ks) {
            const uint64_t o = (uint64_t)(2 * (ks & 3));
            tc_mma_bf16(d, qd + o + (uint64_t)((ks >> 2) * (C::QCHUNK / 16)), kd + o + (uint64_t)((ks >> 2) * (C::KCHUNK / 16)), IDESC_S, ks > 0 ? 1u : 0u);
          }
          tc_commit(s_bar(i));
          if (i == tiles - 1) tc_commit(empty_bar(0, blk));
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
          for (int i = 0; i < tiles && ok; ++i) {
            ok = mbar_wait(h_bar(i), c[i] & 1u, abort_flag);
            if (ok && i == 0) ok = mbar_wait(full_bar(1, g), (g >> 1) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t d = tmem + PT_TM_O + i * 128, pa = tmem + PT_TM_S + i * 128;
            const uint64_t vd = umma_desc_sw128(base + C::O_V + (g & 1u) * C::KTILE);
            if (leader) {
#pragma unroll
              for (int ks = 0; ks < PT_KB / 32; ++ks)
                tc_mma_bf16_ta(d, pa + ks * 8, vd + (uint64_t)((ks >> 2) * (C::VCHUNK / 16) + 2 * (ks & 3)), IDESC_O, (t > 0 || ks > 0) ? 1u : 0u);
            }
            __syncwarp();
            ok = __all_sync(0xffffffffu, mbar_wait(p_bar(i), c[i]++ & 1u, abort_flag));
            if (!ok) break;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int ks = PT_KB / 32; ks < PT_KB / 16; ++ks)
                tc_mma_bf16_ta(d, pa + ks * 8, vd + (uint64_t)((ks >> 2) * (C::VCHUNK / 16) + 2 * (ks & 3)), IDESC_O, 1u);
              tc_commit(o_bar(i));
              if (i == tiles - 1) tc_commit(empty_bar(1, g));
            }
            __syncwarp();
            if (t + 1 < W.nb) ok = scores(i, g + 1, tiles);       // over the probabilities just multiplied: the pipe keeps the order
          }
        }
      }
    }
  } else {
    // ------------------------------ softmax ------------------------------
    const int i = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t tS = tmem + PT_TM_S + i * 128 + lane_addr, tO = tmem + PT_TM_O + i * 128 + lane_addr;
    PtWalk W;
    W.begin(L);
    uint32_t g = 0, c = 0;                   // blocks of the CTA, of this tile
    bool dead = false;
    while (W.next(L, P)) {                   // (none in an idle CTA)
      if (W.pair * PT_ROWS + i * 128 >= R) { g += W.nb; continue; }           // the item has one tile
      const int rr = W.pair * PT_ROWS + i * 128 + row;
      const bool valid = rr < R;
      const int qi = valid ? rr / P.group : 0, hd = valid ? rr - qi * P.group : 0;
      const int len = min(L.len[W.b], cap), keys = min(len + P.n_new, cap);
      unsigned long long word = row_word(P, W.b, qi);
      // queries, coalesced: the warp's 32 rows, 32 * 8 / DH of them per instruction, scaled into fp16's range, into shared memory (the
      // tile's last scores have been formed: this thread waited for them); rows behind the last one hold some real row and
      // are worked on, but not written
      constexpr int PIECES = DH / 8, RPI = 32 / PIECES;
      const int piece = lane % PIECES;
      float down;                            // what this row's queries were divided by
      {
        const long long off = ((long long)W.b * P.n + qi) * P.q_stride + (long long)(W.h * P.group + hd) * DH;
#pragma unroll 1
        for (int u = 0; u < PIECES; ++u)
          cp_async16(base + i * C::QTILE + pt_q_off(quad * 32 + u * RPI + lane / PIECES, piece),
                     reinterpret_cast<const uint4*>((const bf16*)P.q + __shfl_sync(0xffffffffu, off, u * RPI + lane / PIECES)) + piece, true);
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
        // this thread's own row, in place
        uint32_t top = 0u;
#pragma unroll 4
        for (int c8 = 0; c8 < PIECES; ++c8) top = abs2_max(top, *reinterpret_cast<const uint4*>(bp + i * C::QTILE + pt_q_off(row, c8)));
        float up;
        p8_range(__uint_as_float(max(top & 0xffffu, top >> 16) << 16), up, down);
#pragma unroll 2
        for (int c8 = 0; c8 < PIECES; ++c8) {
          uint4* at = reinterpret_cast<uint4*>(bp + i * C::QTILE + pt_q_off(row, c8));
          float f[8];
          bf16x8_to_float(*at, f);
          *at = make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up), pack_f16(f[6] * up, f[7] * up));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        mbar_arrive(q_bar(i));
      }
      if (!valid) word = 0ull;
      float m_ref = -INFINITY, l_run = 0.f, vref = 1.f;
      for (int t = 0; t < W.nb; ++t, ++g, ++c) {
        if (!dead) dead = __any_sync(0xffffffffu, !mbar_wait(table_bar(g), (g >> 2) & 1u, abort_flag) || !mbar_wait(s_bar(i), c & 1u, abort_flag));
        if (dead) continue;
        tc_fence_after();
        const P8Table* tab = tabs + (g & 3u);
        const long long k0 = (long long)(W.t0 + t) * PT_KB;
        const uint4 lv = *reinterpret_cast<const uint4*>(tab->live);
        const bool masked = k0 + PT_KB > len || (lv.x & lv.y & lv.z & lv.w) != 0xffffffffu;
        unsigned long long vis[2] = {~0ull, ~0ull};
        if (masked) {
          vis[0] = row_bits(word, k0, len, keys) & ((unsigned long long)lv.y << 32 | lv.x);
          vis[1] = row_bits(word, k0 + 64, len, keys) & ((unsigned long long)lv.w << 32 | lv.z);
        }
        vref = tab->vref;
        // The block's scores in quarters of 32, so that they stay in registers: for their maximum, and again for their probabilities,
        // which lie, two to a column, over the lower half's scores. The quarters are a loop: unrolled, the kernel's code was more than
        // the instruction cache holds (a quarter of its requests missed, and warps waited for instructions as long as for data).
        constexpr int AT = P8T_AT;           // scores at a time
        float s[AT];
        float m_blk = -INFINITY, widest = 0.f;
        const bool zero = masked && p8t_mask(tS, tab, vis[0], vis[1], down * P.scale_log2);
#pragma unroll 1
        for (int part = 0; part < PT_KB / AT; ++part) {
          tc_ld32(tS + part * AT, s);
          float ks[AT / 16];
#pragma unroll
          for (int b = 0; b < AT / 16; ++b) ks[b] = tab->ks[part * (AT / 16) + b];
#pragma unroll
          for (int b = 0; b < AT / 16; ++b) {
            const float* x = s + 16 * b;
            const float m0 = max3_nan(x[0], x[1], x[2]), m1 = max3_nan(x[3], x[4], x[5]), m2 = max3_nan(x[6], x[7], x[8]), m3 = max3_nan(x[9], x[10], x[11]);
            const float mx = max3_nan(max3_nan(m0, m1, m2), max3_nan(x[12], x[13], x[14]), max3_nan(m3, x[15], x[15]));
            const float kd = ks[b] * down;
            widest = fmaxf(widest, kd);
            m_blk = max3_nan(m_blk, mx == -INFINITY ? mx : __fmul_rn(mx, kd), -INFINITY);
          }
        }
        float f = 1.f;
        if (m_ref == -INFINITY) {
          m_ref = m_blk;                     // nothing has been added for this row yet
        } else if ((m_blk - m_ref) * P.scale_log2 > TC_RESCALE_LOG2) {
          f = ex2_approx((m_ref - m_blk) * P.scale_log2);
          m_ref = m_blk;
          l_run *= f;
        }
        f *= tab->fv;
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
        // scale * (score - reference) + log2 r as one multiply-add, product * (scales) - (scale * reference - log2 r). The latter is
        // rounded, half a unit of its last place off: a common factor of a row's 16 probabilities, below 2^0.5 while it is below 2^24.
        // From there on (or where a factor leaves fp32) the difference is taken first.
        const float scaled = __fmul_rn(sub, P.scale_log2);
        if (__any_sync(0xffffffffu, fabsf(scaled) >= 16777216.f || !(widest * P.scale_log2 < 1e30f) || zero)) {
          l_run += p8t_slow(tS, tab, down, sub, P.scale_log2);
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          tc_fence_before();
          mbar_arrive(h_bar(i));
        } else {
          const float dsc = down * P.scale_log2;
#pragma unroll 1
          for (int part = 0; part < PT_KB / AT; ++part) {
            tc_ld32(tS + part * AT, s);
            float ks[AT / 16], lr[AT / 16], ir[AT / 16];
#pragma unroll
            for (int b = 0; b < AT / 16; ++b) { ks[b] = tab->ks[part * (AT / 16) + b]; lr[b] = tab->lr[part * (AT / 16) + b]; ir[b] = tab->ir[part * (AT / 16) + b]; }
#pragma unroll
            for (int b = 0; b < AT / 16; ++b) {
              const float cs = ks[b] * dsc, off = lr[b] - scaled;
              const uint64_t cs2 = f2_pack(cs, cs), off2 = f2_pack(off, off);
              uint64_t l2 = 0ull;
              uint32_t w8[8];
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                float p0, p1;
                f2_unpack(f2_fma(f2_pack(s[16 * b + 2 * u], s[16 * b + 2 * u + 1]), cs2, off2), p0, p1);
                p0 = ex2_approx(p0);
                p1 = ex2_approx(p1);
                l2 = f2_add(l2, f2_pack(p0, p1));
                w8[u] = pack_f16(p0, p1);
              }
              tc_st8(tS + (uint32_t)(part * (AT / 2) + b * 8), w8);
              float a0, a1;
              f2_unpack(l2, a0, a1);
              l_run = fmaf(a0 + a1, ir[b], l_run);
            }
            if (part == PT_KB / AT / 2 - 1) {
              asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
              tc_fence_before();
              mbar_arrive(h_bar(i));
            }
          }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        mbar_arrive(p_bar(i));
      }
      // ---- the segment's result ----
      if (!dead) dead = __any_sync(0xffffffffu, !mbar_wait(o_bar(i), (c - 1u) & 1u, abort_flag));
      tc_fence_after();
      __threadfence_block();
      if (__any_sync(0xffffffffu, *odd_flag != 0 && !dead)) p8t_add_odd<DH>(P, W.b, W.h, (long long)W.t0 * PT_KB, (long long)(W.t0 + W.nb) * PT_KB, len, keys, word, tO);
      const bool none = (l_run == 0.f || word == 0ull) && !dead;     // the row sees nothing
      const float inv = dead ? __int_as_float(0x7fffffff) : none ? 0.f : vref / l_run;
      const size_t piece_at = (size_t)blockIdx.x * 2 + (W.x0 > W.x_begin ? 1 : 0), prow = piece_at * PT_ROWS + i * 128 + row;
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
          const float unit = none ? 0.f : vref * P8_PIECE;
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(P.part_o + ((piece_at * (DH / 4) + (d + e) / 4) * PT_ROWS + i * 128 + row) * 4) =
                none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[e] * unit, o[e + 1] * unit, o[e + 2] * unit, o[e + 3] * unit);
        }
      }
      if (W.whole) {                         // coalesced, as the queries came
        const long long off = valid ? (((long long)W.b * P.n + qi) * P.hq + W.h * P.group + hd) * DH : -1ll;
        __syncwarp();
#pragma unroll 2
        for (int u = 0; u < PIECES; ++u) {
          const long long o = __shfl_sync(0xffffffffu, off, u * RPI + lane / PIECES);
          if (o >= 0)
            *reinterpret_cast<uint4*>((bf16*)P.out + o + piece * 8) =
                *reinterpret_cast<const uint4*>(bp + i * C::QTILE + pt_q_off(quad * 32 + u * RPI + lane / PIECES, piece));
        }
        __syncwarp();
      }
      if (!W.whole && valid) {
        P.part_ml[prow * 2] = none ? -INFINITY : m_ref;
        P.part_ml[prow * 2 + 1] = dead ? __int_as_float(0x7fffffff) : none ? 0.f : l_run * P8_PIECE;
      }
      tc_fence_before();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace moa
