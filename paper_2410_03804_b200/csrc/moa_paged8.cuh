// A paged key / value cache in 8 bits, a scale for each block of 16 positions and head, and the attention of a few rows over it
// (sm_100a).
//
//   scale = max |x| / 127 over the block's 16 x head_dim values of a head, code = round(x * (127 / max)),  x ~ code * scale
//   s_j = scale * q . k_j,  out = sum_j softmax(s)_j v_j,  as in moa_paged.cuh
//
// When values are rounded: a block is closed, all 16 rows at once, when its last row is committed. Until then its rows, and the
// rows that are not committed, lie in 16 bits in a ring of 80 rows per sequence (slot % 80: an open block and 64 new rows). So a
// row is rounded once, by the scale of the rows it stays with, and a tree's rejected rows never reach a scale.
//
// A closed block of a head is one record of 32 * head_dim + 16 bytes: the keys' codes, the values' codes, the two scales. One bulk
// copy brings what a warp needs for 16 positions. Codes are stored plus 128, in the order in which the tensor cores' operands want
// them, so that a lane's 16 bytes are loaded whole, without bank conflicts, and become operand registers by byte masks:
//   keys    (token % 2, dim / 64, token / 2, dim % 64): 16 dims of a token are 16 bytes
//   values  (dim / 32, dim % 8, token / 4, dim / 8 % 4, token % 4): 4 tokens of a dim are a word
// 8-bit codes become fp16, exactly, by placing the byte under the exponent of 1024 and subtracting 1152: two instructions for two codes.
// (A byte with zeros above it is (code + 128) * 2^-24 already, but taking the 128 off the sums afterwards -- from scores by the query's
// sum, from outputs by one more product of a constant per block -- cost precision where sums cancel and gained nothing.) Queries are
// scaled by a power of two per row into fp16's range (exact for what lies within 2^31 of the row's largest).
//
// What bounds it: one token reads a byte and 1/16 of a scale per cached value once, so the cache's stream from HBM does. 256 bytes
// per position and head leave 175 cycles of an SM per 16 positions and head, 700 instructions. A short cache is bound by the chain of
// its steps instead: the lengths, the work's line, the first copies, the join.
// Measured, one token of 32 heads over 8, head_dim 128: over 2047 positions 11.5 us, over 32767 24.1 us, 16 sequences of up to 8192
// 42.8 us (the caches alone at a copy's rate: 0.6, 10.2 and 26.4). Appending 2 x 8 heads of 2043 rows and reading them back 14.6 us in
// a graph, 12.6 to 13.0 among other calls.
#pragma once
#include <cuda_fp16.h>

#include "moa_paged.cuh"
#include "moa_wstream.cuh"

namespace moa {

constexpr int P8_BLOCK = 16;                 // positions that share a scale
constexpr int P8_RING = 80;                  // rows of the 16-bit ring: 15 of an open block + 64 new ones, in whole blocks
constexpr int P8_STAGES = 2;
constexpr float P8_BIAS = 7.f;               // probabilities enter their fp16 product times 2^7: a row's maximum may pass the
constexpr float P8_LAZY = 8.f;               // reference by 2^8 before the sums move to a new one, and 2^15 fits fp16
// Sums and outputs of a piece are handed on times 2^-16 beside that: probabilities times values are divided at the very end only, and
// values may be bf16's largest while a row's probabilities, in units of the largest, sum up to no more than 2^16 (values up to 2^106: as
// long as there are positions). The room comes off the other end: outputs below 2^-110, far under a closed block's least, lose bits.
constexpr float P8_PIECE = 0x1p-23f;         // 2^-P8_BIAS * 2^-16
constexpr int P8_OPEN = 100;                 // log2 of the open rows' values over the unit of the outputs, at most
constexpr int P8_LEAST = -105;               // log2 of the least unit: scales are 0 or above 2^-107, units 4 to 8 times those

template <int DH> struct P8Cfg {
  static constexpr int CODES = P8_BLOCK * DH;                   // of the keys, and of the values
  static constexpr int REC = 2 * CODES + 16;
  static constexpr int SCRATCH = 16 * DH * 2;                   // of one warp: 16 rows of 16-bit values, or its merged output
  static constexpr int SMEM = PG_WARPS * (P8_STAGES * REC + SCRATCH);
  static_assert(PG_ROWS * DH * 4 <= SCRATCH, "a warp's output fits its scratch");
};

struct Paged8 {
  PagedAttn a;                               // a.c.k, a.c.v: the rings, bf16 [batch, P8_RING, hkv, DH]; its pages and weights are not used
  const uint8_t* pages;                      // [n_pages, hkv, page_size / 16] records, pages page_bytes apart
  long long page_bytes;
  uint8_t* open;                             // open blocks as the tree kernel wants them (moa_paged8_tc.cuh)
};

// The record of block blk of (sequence, head), or null where the table has no such page.
template <int DH>
__device__ __forceinline__ const uint8_t* p8_record(const PagedView& c, const uint8_t* pages, long long page_bytes, int b, int h, int blk) {
  const int per = c.shift - 4, page = c.table[(size_t)b * c.max_pages + (blk >> per)];
  if (page < 0 || page >= c.n_pages) return nullptr;
  return pages + page * page_bytes + (long long)((h << per) + (blk & ((1 << per) - 1))) * P8Cfg<DH>::REC;
}
__device__ __forceinline__ size_t p8_ring_row(const PagedView& c, int b, int slot, int h, int dh) {
  return (((size_t)b * P8_RING + slot % P8_RING) * c.hkv + h) * (size_t)dh;
}

// ---------------------------------------------------------------------------------------------
// Closing blocks
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t abs2_max(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }
__device__ __forceinline__ uint32_t abs2_max(uint32_t m, const uint4& x) { return abs2_max(abs2_max(abs2_max(abs2_max(m, x.x), x.y), x.z), x.w); }

// Largest finite |x| of packed bf16 patterns, kept packed.
__device__ __forceinline__ uint32_t finite2_max(uint32_t m, uint32_t w) {
  w = odd_cleared(w) & 0x7fff7fffu;
  return __vmaxu2(m, w);
}
__device__ __forceinline__ uint32_t finite2_max(uint32_t m, const uint4& x) { return finite2_max(finite2_max(finite2_max(finite2_max(m, x.x), x.y), x.z), x.w); }

struct P8Scale {
  float scale, inv;                          // of the record, and codes per unit
  // top: largest |x| as a bf16 pattern. A block with a value that is not finite has scale NaN, so that who sees it gets NaN; one whose
  // values are all below 2^-100 is held as zeros (127 / max would leave fp32 from 2^-121 on).
  __device__ __forceinline__ explicit P8Scale(uint32_t top) {
    const float m = __uint_as_float(top << 16);
    const bool odd = top >= 0x7f80u, none = m < 0x1p-100f;
    scale = odd ? __int_as_float(0x7fffffff) : none ? 0.f : m / 127.f;
    inv = odd || none ? 0.f : 127.f / m;
  }
  // code + 128 in the low byte; the product is rounded to fp32, then to an integer, ties to even. |x * inv| < 127.5.
  __device__ __forceinline__ uint32_t code(float x) const {
    return __float_as_uint(__fadd_rn(inv == 0.f ? 0.f : __fmul_rn(x, inv), 12582912.f + 128.f));
  }
  __device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) const {
    return __byte_perm(__byte_perm(code(a), code(b), 0x0040), __byte_perm(code(c), code(d), 0x0040), 0x5410);
  }
};

// One warp closes one block of one head. src(t): row t's head in k or v, bf16, 16-byte aligned.
template <int DH, typename Src>
__device__ __forceinline__ void p8_close(uint8_t* rec, Src src) {
  const int lane = threadIdx.x & 31;
  float ks, vs;
  {                                          // keys: a lane takes 16 dims of tokens 2 gq and 2 gq + 1
    const int gq = lane >> 2, tq = lane & 3;
    uint4 x[2][DH / 64][2];
    uint32_t top = 0u;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint4* r = reinterpret_cast<const uint4*>(src(0, 2 * gq + p));
#pragma unroll
      for (int k = 0; k < DH / 64; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) x[p][k][e] = __ldcg(r + k * 8 + tq * 2 + e);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < DH / 64; ++k) top = abs2_max(abs2_max(top, x[p][k][0]), x[p][k][1]);
    const P8Scale S(__reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16)));
    ks = S.scale;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < DH / 64; ++k) {
        float f[16];
        bf16x8_to_float(x[p][k][0], f);
        bf16x8_to_float(x[p][k][1], f + 8);
        *reinterpret_cast<uint4*>(rec + (p * (DH / 64) + k) * 512 + lane * 16) =
            make_uint4(S.code4(f[0], f[1], f[2], f[3]), S.code4(f[4], f[5], f[6], f[7]), S.code4(f[8], f[9], f[10], f[11]), S.code4(f[12], f[13], f[14], f[15]));
      }
  }
  {                                          // values: a lane takes 8 dims of tokens 4 tq .. 4 tq + 3
    const int tq = lane & 3, c = lane >> 2;
    uint4 x[DH / 64][4];
    uint32_t top = 0u;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint4* r = reinterpret_cast<const uint4*>(src(1, 4 * tq + t));
#pragma unroll
      for (int u = 0; u < DH / 64; ++u) x[u][t] = __ldcg(r + u * 8 + c);
    }
#pragma unroll
    for (int u = 0; u < DH / 64; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t) top = abs2_max(top, x[u][t]);
    const P8Scale S(__reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16)));
    vs = S.scale;
#pragma unroll
    for (int u = 0; u < DH / 64; ++u) {
      const int d8 = u * 8 + c;              // dim / 8
      float f[4][8];
#pragma unroll
      for (int t = 0; t < 4; ++t) bf16x8_to_float(x[u][t], f[t]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<uint32_t*>(rec + P8Cfg<DH>::CODES + (d8 >> 2) * 512 + e * 64 + tq * 16 + (d8 & 3) * 4) = S.code4(f[0][e], f[1][e], f[2][e], f[3][e]);
    }
  }
  if (lane == 0) *reinterpret_cast<float2*>(rec + 2 * P8Cfg<DH>::CODES) = make_float2(ks, vs);
}

// Rows of a prompt behind the committed ones: closes every block that becomes whole, keeps the rest in the ring. A warp per
// (sequence, block, head); the one of a sequence's first block reads the open rows before it writes the rows that stay open, whose
// places in the ring may be theirs.
template <int DH>
__global__ void __launch_bounds__(256) paged8_append_kernel(const PagedView C, uint8_t* pages, long long page_bytes, const bf16* k_new,
                                                            const bf16* v_new, long long row_stride, int n, const int* n_new, int blocks) {
  pdl_trigger();
  pdl_wait(KID_APPEND);
  const int b = blockIdx.y, lane = threadIdx.x & 31;
  const int len = C.len[b];
  if (len < 0) return;
  const long long cap = C.cap();
  const int rows = n_new ? max(0, min(n, n_new[b])) : n;
  const int end = (int)min((long long)len + rows, cap), base = len >> 4, n_close = (end >> 4) - base;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < (long long)blocks * C.hkv; w += (long long)gridDim.x * 8) {
    const int j = (int)(w / C.hkv), h = (int)(w - (long long)j * C.hkv);
    if (j > 0 && j >= n_close) break;
    auto src = [&](int kv, int t) -> const bf16* {
      const int slot = ((base + j) << 4) + t;
      if (slot < len) return (const bf16*)(kv ? C.v : C.k) + p8_ring_row(C, b, slot, h, DH);
      return (kv ? v_new : k_new) + ((long long)b * n + (slot - len)) * row_stride + (long long)h * DH;
    };
    if (j < n_close) {
      uint8_t* rec = const_cast<uint8_t*>(p8_record<DH>(C, pages, page_bytes, b, h, base + j));
      if (rec) p8_close<DH>(rec, src);
    }
    if (j == 0) {                            // rows that stay open
      __syncwarp();
      constexpr int PIECES = DH / 8;
      const int first = max(len, (end >> 4) << 4);
      for (int i = lane; i < (end - first) * PIECES * 2; i += 32) {
        const int kv = i & 1, p = (i >> 1) % PIECES, slot = first + (i >> 1) / PIECES;
        const uint4 x = __ldcg(reinterpret_cast<const uint4*>((kv ? v_new : k_new) + ((long long)b * n + (slot - len)) * row_stride + (long long)h * DH) + p);
        reinterpret_cast<uint4*>((bf16*)(kv ? C.v : C.k) + p8_ring_row(C, b, slot, h, DH))[p] = x;
      }
    }
  }
}

// Keeps the accepted path of n uncommitted rows (slot len + acc_slot[j] moves to slot len + j, j < acc_len; without acc_slot the
// rows stay where they are) and closes the blocks that become whole. A CTA per (sequence, head); a warp per closed block. The
// path's rows are all read before one is written.
template <int DH>
__global__ void __launch_bounds__(256) paged8_commit_kernel(const PagedView C, uint8_t* pages, long long page_bytes, int n, const int* acc_slot,
                                                            const int* acc_len, int cap) {
  pdl_trigger();
  pdl_wait();
  constexpr int PIECES = DH / 8, MAXV = 64 * PIECES / 256;
  const int h = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5;
  const int len = C.len[b];
  if (len < 0) return;
  __shared__ int s_n, s_slot[64];
  const int most = (int)min((long long)n, C.cap() - len);
  if (threadIdx.x == 0) {
    int m = max(0, min(min(acc_len ? acc_len[b] : n, acc_slot ? cap : n), most));
    if (acc_slot) {
      int last = -1, j = 0;
      for (; j < m; ++j) {
        const int s = acc_slot[(size_t)b * cap + j];
        if (s <= last || s >= most) break;
        s_slot[j] = last = s;
      }
      for (int i = j; i < m; ++i) s_slot[i] = i;                     // entries that do not rise end the path's moves
    }
    s_n = m;
  }
  __syncthreads();
  const int m = s_n;
  if (acc_slot) {
    uint4 rk[MAXV], rv[MAXV];
#pragma unroll
    for (int u = 0; u < MAXV; ++u) {
      const int i = threadIdx.x + u * 256, j = i / PIECES, c = i - j * PIECES;
      if (j < m && s_slot[j] != j) {
        const size_t at = p8_ring_row(C, b, len + s_slot[j], h, DH) / 8 + c;
        rk[u] = reinterpret_cast<const uint4*>(C.k)[at];
        rv[u] = reinterpret_cast<const uint4*>(C.v)[at];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MAXV; ++u) {
      const int i = threadIdx.x + u * 256, j = i / PIECES, c = i - j * PIECES;
      if (j < m && s_slot[j] != j) {
        const size_t at = p8_ring_row(C, b, len + j, h, DH) / 8 + c;
        reinterpret_cast<uint4*>(C.k)[at] = rk[u];
        reinterpret_cast<uint4*>(C.v)[at] = rv[u];
      }
    }
    __threadfence_block();
    __syncthreads();
  }
  const int base = len >> 4, n_close = ((len + m) >> 4) - base;      // at most 4
  if (warp >= n_close) return;
  uint8_t* rec = const_cast<uint8_t*>(p8_record<DH>(C, pages, page_bytes, b, h, base + warp));
  if (rec) p8_close<DH>(rec, [&](int kv, int t) { return (const bf16*)(kv ? C.v : C.k) + p8_ring_row(C, b, ((base + warp) << 4) + t, h, DH); });
}

// Rows t0 .. t1 - 1 of a closed block of which the first `rows` are wanted; the others, and all of a missing page's, are zeros.
// k_out, v_out: where the block's row 0 would go, rows ld elements apart.
template <typename T, int DH>
__device__ __noinline__ void p8_read_part(const uint8_t* rec, int rows, int t0, int t1, T* k_out, T* v_out, int ld) {
  const float2 scale = rec ? __ldcg(reinterpret_cast<const float2*>(rec + 2 * P8Cfg<DH>::CODES)) : make_float2(0.f, 0.f);
  for (int t = t0; t < t1; ++t)
    for (int d = threadIdx.x & 31; d < DH; d += 32) {
      float x = 0.f, y = 0.f;
      if (rec && t < rows) {
        x = (float)(rec[((t & 1) * (DH / 64) + d / 64) * 512 + (t >> 1) * 64 + d % 64] - 128) * scale.x;
        y = (float)(rec[P8Cfg<DH>::CODES + d / 32 * 512 + d % 8 * 64 + (t >> 2) * 16 + d / 8 % 4 * 4 + (t & 3)] - 128) * scale.y;
      }
      T *k = k_out + (long long)t * ld + d, *v = v_out + (long long)t * ld + d;
      if constexpr (sizeof(T) == 2) { *k = __float2bfloat16_rn(x); *v = __float2bfloat16_rn(y); }
      else { *k = x; *v = y; }
    }
}

// Rows first[b] + i, i < n, of the cache's first length[b] rows, [batch, n, hkv, DH]: a warp per (sequence, block, head). A layer that has
// not been advanced yet has more rows than its len says; with fewer, the last block may be a closed one of which only a part is wanted.
template <typename T, int DH>
__global__ void __launch_bounds__(256) paged8_read_kernel(const PagedView C, const uint8_t* pages, long long page_bytes, int n, const int* first,
                                                          const int* length, T* k_out, T* v_out, int blocks) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y, lane = threadIdx.x & 31;
  const int shut = C.len[b];
  if (shut < 0 || length[b] < 0) return;
  const int len = (int)min((long long)length[b], C.cap());
  const long long f = first ? first[b] : 0;
  const int b0 = (int)((f >= 0 ? f : f - 15) / 16);
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < (long long)blocks * C.hkv; w += (long long)gridDim.x * 8) {
    const int j = (int)(w / C.hkv), h = (int)(w - (long long)j * C.hkv);
    const long long s0 = ((long long)b0 + j) * 16, i0 = s0 - f;      // the block's first slot, and where it would go
    if (i0 >= n) break;
    const uint8_t* rec = nullptr;
    float2 scale = make_float2(0.f, 0.f);
    if (s0 >= 0 && s0 + 16 <= len) rec = p8_record<DH>(C, pages, page_bytes, b, h, (int)(s0 >> 4));
    if (rec) scale = __ldcg(reinterpret_cast<const float2*>(rec + 2 * P8Cfg<DH>::CODES));
    const bool open = s0 >= 0 && s0 < len && s0 + 16 > len;
    auto put = [&](T* out, int t, int d, const float* x) {           // 8 values
      const long long i = i0 + t;
      if (i < 0 || i >= n) return;
      T* to = out + (((size_t)b * n + i) * C.hkv + h) * DH + d;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
      } else {
        reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
      }
    };
    // a byte under the exponent of 2^23, less that and 128 (conversions of integers run at a quarter of this rate)
    auto byte = [](uint32_t w4, int e) { return __uint_as_float(__byte_perm(w4, 0x4b000000u, 0x7540 | e)) - 8388736.f; };
    const int gq = lane >> 2, tq = lane & 3;
    if (rec) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < DH / 64; ++k) {
          const uint4 c = __ldcg(reinterpret_cast<const uint4*>(rec + (p * (DH / 64) + k) * 512) + lane);
          const uint32_t w4[4] = {c.x, c.y, c.z, c.w};
          float x[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = byte(w4[e >> 2], e & 3) * scale.x;
          put(k_out, 2 * gq + p, k * 64 + tq * 16, x);
          put(k_out, 2 * gq + p, k * 64 + tq * 16 + 8, x + 8);
        }
#pragma unroll
      for (int u = 0; u < DH / 64; ++u) {
        const int d8 = u * 8 + gq;
        uint32_t w4[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w4[e] = __ldcg(reinterpret_cast<const uint32_t*>(rec + P8Cfg<DH>::CODES + (d8 >> 2) * 512 + e * 64 + tq * 16 + (d8 & 3) * 4));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = byte(w4[e], t) * scale.y;
          put(v_out, 4 * tq + t, d8 * 8, x);
        }
      }
      continue;
    }
    if (open && s0 + 16 <= min((long long)shut, C.cap())) {          // (rare) a part of a block that is closed
      const long long at = (((long long)b * n + i0) * C.hkv + h) * DH;
      p8_read_part<T, DH>(p8_record<DH>(C, pages, page_bytes, b, h, (int)(s0 >> 4)), (int)(len - s0), (int)max(0ll, -i0), (int)min(16ll, n - i0), k_out + at, v_out + at,
                          C.hkv * DH);
      continue;
    }
    for (int i = lane; i < 16 * (DH / 8); i += 32) {                 // the open block, or no row at all
      const int t = i / (DH / 8), d = i % (DH / 8) * 8;
      float x[8], y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
      if (open && s0 + t < len) {
        const size_t at = (p8_ring_row(C, b, (int)s0 + t, h, DH) + d) / 8;
        bf16x8_to_float(reinterpret_cast<const uint4*>(C.k)[at], x);
        bf16x8_to_float(reinterpret_cast<const uint4*>(C.v)[at], y);
      }
      put(k_out, t, d, x);
      put(v_out, t, d, y);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Attention of a few query rows. Work split, pieces and their join are those of the paged row kernel (moa_paged.cuh), with two CTAs per
// SM: while one merges its warps at the end of an item, the other's copies go on.
// A long axis is cut into no more pieces than pay for their join: it costs the CTA that makes it about a tenth of a tile's time each, so
// pieces of sqrt(T / 10) tiles balance both. One head over 30000 positions 17.0 us (26.0 with pieces of one tile, 18.9 and 18.5 with
// sqrt(T / 5) and sqrt(T / 20)), over 100000 25.2 (32.6); where the heads fill the GPU nothing changes (8 over 32767: 21.3).
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_f16_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Two codes (plus 128), each under the exponent of fp16's 1024, as what they stand for.
__device__ __forceinline__ uint32_t p8_less_bias(uint32_t w) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x64806480u));          // 1024 + 128
  return r;
}
// Four codes (plus 128) of a word as what they stand for: bytes 0 and 2, bytes 1 and 3.
__device__ __forceinline__ void p8_codes(uint32_t w, uint32_t& even, uint32_t& odd) {
  even = p8_less_bias((w & 0x00ff00ffu) | 0x64006400u);
  odd = p8_less_bias(__byte_perm(w, 0x64646464u, 0x4341));
}
// Power of two that brings a row whose largest |x| is m to at most 2^15, and its inverse; 1 for a row without a finite largest.
__device__ __forceinline__ void p8_range(float m, float& up, float& down) {
  const int e = (int)(__float_as_uint(m) >> 23);                     // biased exponent
  const bool fit = e > 15 && e < 255;
  up = fit ? __uint_as_float((uint32_t)(127 + 14 + 127 - e) << 23) : 1.f;          // 2^(14 - (e - 127)), e - 127 >= -111
  down = fit ? __uint_as_float((uint32_t)(e - 14) << 23) : 1.f;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// One warp's running state over 8 query rows. Maxima are of unscaled scores; sums and outputs are times 2^P8_BIAS, outputs in
// units of vref, a power of two that only rises: above the scales of the closed blocks that it has met, so that their probabilities
// times scales fit fp16, and at most 2^P8_OPEN below the open rows' values, which enter as bf16, so that no sum leaves fp32: up
// to 2^8 (P8_LAZY) * 2^7 * 16 rows * 2^P8_OPEN. It lies that far below them so that open values take no bits off closed blocks of
// much smaller ones, which rows that do not see the open values still want to the last.
template <int DH>
struct Paged8Warp {
  static constexpr int KS = DH / 16;
  uint32_t qf[KS][2];                        // query gq: dims 64 c + 16 tq + 4 j + {0, 2}, {1, 3} of k-step 4 c + j
  float o[DH / 16][4];                       // columns 16 d + gq and + 8 of queries 2 tq and 2 tq + 1
  float m[2], l[2], qd[2];                   // queries 2 tq, 2 tq + 1: reference, sum over this lane's positions, scale of its fp16 form
  float vref, inv_vref;
  unsigned long long word[2];                // their mask words
  int gq, tq;

  static __device__ __forceinline__ const bf16* q_row(const PagedAttn& P, int b, int h, int mt, int gq) {
    const int R = P.n * P.group, r = mt * PG_ROWS + gq, rc = r < R ? r : 0;        // queries behind the last one are worked on and not written
    return (const bf16*)P.q + ((long long)b * P.n + rc / P.group) * P.q_stride + (long long)(h * P.group + rc % P.group) * DH;
  }
  __device__ __forceinline__ void begin(const PagedAttn& P, int b, int h, int mt) {
    const int lane = threadIdx.x & 31, R = P.n * P.group;
    gq = lane >> 2; tq = lane & 3;
    const uint4* src = reinterpret_cast<const uint4*>(q_row(P, b, h, mt, gq));
    uint4 x[DH / 64][2];
#pragma unroll
    for (int c = 0; c < DH / 64; ++c)
#pragma unroll
      for (int e = 0; e < 2; ++e) x[c][e] = src[c * 8 + tq * 2 + e];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int rr = mt * PG_ROWS + 2 * tq + u;
      word[u] = rr < R ? row_word(P, b, rr / P.group) : 0ull;
    }
    uint32_t top = 0u;
#pragma unroll
    for (int c = 0; c < DH / 64; ++c) top = abs2_max(abs2_max(top, x[c][0]), x[c][1]);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float up, down;
    p8_range(__uint_as_float(top << 16), up, down);
#pragma unroll
    for (int c = 0; c < DH / 64; ++c) {
      float f[16];
      bf16x8_to_float(x[c][0], f);
      bf16x8_to_float(x[c][1], f + 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        qf[c * 4 + j][0] = pack_f16(f[4 * j] * up, f[4 * j + 2] * up);
        qf[c * 4 + j][1] = pack_f16(f[4 * j + 1] * up, f[4 * j + 3] * up);
      }
    }
    qd[0] = __shfl_sync(0xffffffffu, down, 8 * tq);
    qd[1] = __shfl_sync(0xffffffffu, down, 8 * tq + 4);
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    vref = inv_vref = 0.f;                   // none yet
  }

  // References that the scores z [position][query] have outgrown move up. Rare.
  __device__ __forceinline__ void refer(const PagedAttn& P, const float (*z)[2]) {
    const float z0 = fmaxf(z[0][0], z[1][0]), z1 = fmaxf(z[0][1], z[1][1]);
    if (!__any_sync(0xffffffffu, (z0 - m[0]) * P.scale_log2 > P8_LAZY || (z1 - m[1]) * P.scale_log2 > P8_LAZY)) return;
    float f[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float mx = u ? z1 : z0;
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const float mn = fmaxf(m[u], mx);
      f[u] = mn == m[u] ? 1.f : ex2_approx((m[u] - mn) * P.scale_log2);            // m = -inf: 0
      m[u] = mn;
      l[u] *= f[u];
    }
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) { o[i][0] *= f[0]; o[i][1] *= f[1]; o[i][2] *= f[0]; o[i][3] *= f[1]; }
  }
  // Outputs move to units of `ref`, a power of two. (A factor below fp32's least goes in two steps: infinity times zero is no number.)
  __device__ __forceinline__ void rescale(float ref, float inv) {
    if (vref != 0.f) {
      const float f = vref * inv;
      const bool deep = f < 0x1p-126f;
      const float f1 = deep ? inv : f, f2 = deep ? vref : 1.f;
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = __fmul_rn(__fmul_rn(o[i][e], f1), f2);
      }
    }
    vref = ref;
    inv_vref = inv;
  }

  // One closed block: its record lies at rec.
  __device__ __forceinline__ void block(const PagedAttn& P, const uint8_t* rec) {
    const int lane = threadIdx.x & 31;
    const float2 scale = *reinterpret_cast<const float2*>(rec + 2 * P8Cfg<DH>::CODES);
    float s[2][4];                           // two chains halve the products' latency
#pragma unroll
    for (int c = 0; c < 2; ++c) s[c][0] = s[c][1] = s[c][2] = s[c][3] = 0.f;
    // rows of the product: row r < 8 is position 2 r, row 8 + r position 2 r + 1
#pragma unroll
    for (int c = 0; c < DH / 64; ++c) {
      const uint4 k0 = *reinterpret_cast<const uint4*>(rec + c * 512 + lane * 16), k1 = *reinterpret_cast<const uint4*>(rec + (DH / 64 + c) * 512 + lane * 16);
      const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t a[4];
        p8_codes(w0[j], a[0], a[2]);
        p8_codes(w1[j], a[1], a[3]);
        mma_f16_16816(s[j & 1], a, qf[c * 4 + j][0], qf[c * 4 + j][1]);
      }
    }
    float z[2][2];                           // [position 2 gq, 2 gq + 1][query 2 tq, 2 tq + 1]
    const float t0 = scale.x * qd[0], t1 = scale.x * qd[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e >> 1][e & 1] = (s[0][e] + s[1][e]) * (e & 1 ? t1 : t0);
    refer(P, z);
    if (!(scale.y <= vref)) {                // the same for the whole warp; 4 to 8 times the scale, so that it is rarely passed
      const uint32_t e = scale.y > 0.f ? (__float_as_uint(scale.y) >> 23) + 3u : 127u;         // (a scale may be NaN)
      rescale(__uint_as_float(e << 23), __uint_as_float((254u - e) << 23));
    }
    const float ratio = scale.y * inv_vref;
    const float sub0 = m[0] == -INFINITY ? 0.f : m[0], sub1 = m[1] == -INFINITY ? 0.f : m[1];
    uint32_t pb[2];                          // right operand: positions 4 tq and 4 tq + 2, 4 tq + 1 and 4 tq + 3 of query gq
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float p0 = ex2_approx(fmaf(z[k][0] - sub0, P.scale_log2, P8_BIAS)), p1 = ex2_approx(fmaf(z[k][1] - sub1, P.scale_log2, P8_BIAS));
      l[0] += p0;
      l[1] += p1;
      pb[k] = mat8_trans(pack_f16(p0 * ratio, p1 * ratio));
    }
#pragma unroll
    for (int k = 0; k < DH / 32; ++k) {
      const uint4 v = *reinterpret_cast<const uint4*>(rec + P8Cfg<DH>::CODES + k * 512 + lane * 16);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t a[4];
        p8_codes(w[2 * i], a[0], a[2]);
        p8_codes(w[2 * i + 1], a[1], a[3]);
        mma_f16_16816(o[2 * k + i], a, pb[0], pb[1]);
      }
    }
  }

  // 16 slots of the ring from slot s0 on, a multiple of 16; V: this warp's scratch. Rows of slots from len on come from the call's new
  // rows when it has them, and go to the ring with them (store). One warp of an item comes here while the others wait for it
  // at the item's end, so addresses are made once and stepped.
  __device__ __forceinline__ void open(const Paged8& PP, int b, int h, int mt, int s0, int len, int keys, unsigned long long any, bool store, uint8_t* V) {
    const PagedAttn& P = PP.a;
    const int lane = threadIdx.x & 31, R = P.n * P.group, old = max(0, min(16, len - s0));       // rows that are committed
    const int slot = s0 + (lane & 15);
    const uint32_t live = __ballot_sync(0xffffffffu, slot < keys && (slot < len || ((any >> (slot - len)) & 1ull) != 0ull)) & 0xffffu;
    auto sees = [&](unsigned long long w, int j) -> bool {
      return ((live >> j) & 1u) != 0u && (j < old ? w != 0ull : ((w >> (s0 + j - len)) & 1ull) != 0ull);
    };
    constexpr int NP = DH / 32, NV = DH / 16, CH = DH / 8;           // pieces of 8 elements: per lane of a key row and of all values; of a row
    const size_t ring_at = p8_ring_row(P.c, b, s0, h, DH);           // (a block does not wrap)
    const long long ring_ld = (long long)P.c.hkv * DH, new_at = ((long long)b * P.n + (s0 - len)) * P.new_stride + (long long)h * DH;
    auto row = [&](int kv, int j) -> const bf16* {
      return j >= old && P.k_new ? (const bf16*)(kv ? P.v_new : P.k_new) + new_at + j * P.new_stride : (const bf16*)(kv ? P.c.v : P.c.k) + ring_at + j * ring_ld;
    };
    // the values by copies, past the registers that the queries' and outputs' states leave
#pragma unroll 2
    for (int j = lane / CH; j < 16; j += 32 / CH)
      cp_async16(smem_u32(V) + tile_off<DH>(j, lane % CH), row(1, j) + (lane % CH) * 8, ((live >> j) & 1u) != 0u);
    cp_async_commit();
    uint4 kx[2][NP], qx[NP], fresh[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const bool there = (live >> (gq + 8 * p)) & 1u;
      const uint4* from = reinterpret_cast<const uint4*>(row(0, gq + 8 * p)) + tq;
#pragma unroll
      for (int i = 0; i < NP; ++i) kx[p][i] = there ? __ldcg(from + 4 * i) : make_uint4(0u, 0u, 0u, 0u);
    }
    const uint4* q = reinterpret_cast<const uint4*>(q_row(P, b, h, mt, gq)) + tq;
#pragma unroll
    for (int i = 0; i < NP; ++i) qx[i] = __ldcg(q + 4 * i);
    // the first new row, for the ring: its keys and values
    uint32_t todo = store ? live & ~((1u << old) - 1u) : 0u;
    const int first = __ffs(todo) - 1;
    if (todo != 0u && lane < CH) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) fresh[kv] = __ldcg(reinterpret_cast<const uint4*>(row(kv, first)) + lane);
    }
    cp_async_wait<0>();
    __syncwarp();
    // values that are not finite go by themselves to the rows that see them; zeros stand for them in the product
    bool odd = false;
    uint32_t top = 0u;                       // largest finite |v|
#pragma unroll 4
    for (int u = 0; u < NV; ++u) {
      const uint4 x = reinterpret_cast<const uint4*>(V)[u * 32 + lane];
      odd = odd || odd_any(x);
      top = finite2_max(top, x);
    }
    odd = __any_sync(0xffffffffu, odd);
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16)) >> 7;          // its biased exponent
    float s[2][4];
#pragma unroll
    for (int c = 0; c < 2; ++c) s[c][0] = s[c][1] = s[c][2] = s[c][3] = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const uint32_t a0[4] = {kx[0][i].x, kx[1][i].x, kx[0][i].y, kx[1][i].y}, a1[4] = {kx[0][i].z, kx[1][i].z, kx[0][i].w, kx[1][i].w};
      mma_bf16_16816(s[0], a0, qx[i].x, qx[i].y);
      mma_bf16_16816(s[1], a1, qx[i].z, qx[i].w);
    }
    float z[2][2];                           // [position gq, gq + 8][query]
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e >> 1][e & 1] = sees(word[e & 1], gq + 8 * (e >> 1)) ? s[0][e] + s[1][e] : -INFINITY;
    refer(P, z);
    {                                        // (the first of the item's blocks: no unit is set yet)
      const uint32_t e = max(top, (uint32_t)(127 + P8_LEAST) + P8_OPEN) - P8_OPEN;
      vref = __uint_as_float(e << 23);
      inv_vref = __uint_as_float((254u - e) << 23);
    }
    if (odd) {                               // (rare)
#pragma unroll 1
      for (int j = 0; j < 16; ++j) {
        const bool y0 = sees(word[0], j), y1 = sees(word[1], j);
        const int r = mt * PG_ROWS + 2 * tq;
#pragma unroll
        for (int e = 0; e < DH / 8; ++e) {
          const float v = __bfloat162float(*reinterpret_cast<const bf16*>(V + tile_off<DH>(j, e) + gq * 2));
          if (odd_f(v) && y0 && r < R) o[e >> 1][2 * (e & 1)] += v;
          if (odd_f(v) && y1 && r + 1 < R) o[e >> 1][2 * (e & 1) + 1] += v;
        }
      }
      __syncwarp();
#pragma unroll
      for (int u = 0; u < NV; ++u) reinterpret_cast<uint4*>(V)[u * 32 + lane] = odd_cleared(reinterpret_cast<const uint4*>(V)[u * 32 + lane]);
      __syncwarp();
    }
    const float sub0 = m[0] == -INFINITY ? 0.f : m[0], sub1 = m[1] == -INFINITY ? 0.f : m[1];       // seen nothing: exp2(-inf - 0) = 0
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float p0 = ex2_approx(fmaf(z[k][0] - sub0, P.scale_log2, P8_BIAS)), p1 = ex2_approx(fmaf(z[k][1] - sub1, P.scale_log2, P8_BIAS));
      l[0] += p0;
      l[1] += p1;
      p0 *= inv_vref;
      p1 *= inv_vref;
      const uint32_t w = pack_bf16(p0, p1);
      hi[k] = mat8_trans(w);
      lo[k] = mat8_trans(pack_bf16(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u)));
    }
    const uint32_t sV = smem_u32(V);
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
      uint32_t v[4];
      ldsm_x4_t(sV + tile_off<DH>((lane & 7) + ((lane >> 4) << 3), d * 2 + ((lane >> 3) & 1)), v[0], v[1], v[2], v[3]);
      mma_bf16_16816(o[d], v, hi[0], hi[1]);
      mma_bf16_16816(o[d], v, lo[0], lo[1]);
    }
    if (lane < CH) {
#pragma unroll 1
      for (bool again = false; todo != 0u; todo &= todo - 1u, again = true) {
        const int j = __ffs(todo) - 1;
        uint4* const to = reinterpret_cast<uint4*>((bf16*)P.c.k + ring_at + j * ring_ld) + lane;
        uint4* const to_v = reinterpret_cast<uint4*>((bf16*)P.c.v + ring_at + j * ring_ld) + lane;
        *to = again ? __ldcg(reinterpret_cast<const uint4*>(row(0, j)) + lane) : fresh[0];
        *to_v = again ? __ldcg(reinterpret_cast<const uint4*>(row(1, j)) + lane) : fresh[1];
      }
    }
    __syncwarp();
  }

  // Leaves (max, sum) of every query in sml [8][2] and the outputs in so [DH][8].
  __device__ __forceinline__ void finish(float* so, float* sml) {
    const float unit = vref * P8_PIECE;
    float f[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = l[u];
      t += __shfl_xor_sync(0xffffffffu, t, 4);
      t += __shfl_xor_sync(0xffffffffu, t, 8);
      t += __shfl_xor_sync(0xffffffffu, t, 16);
      const bool blind = word[u] == 0ull;    // a row that sees nothing, not even the closed blocks
      f[u] = blind || vref == 0.f ? 0.f : unit;
      if (gq == 0) { sml[(2 * tq + u) * 2] = blind ? -INFINITY : m[u]; sml[(2 * tq + u) * 2 + 1] = blind ? 0.f : t * P8_PIECE; }
      if (f[u] == 0.f) {                     // (what is there may not be finite)
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) o[i][u] = o[i][2 + u] = 0.f;
      }
    }
    float* at = so + gq * 8 + 2 * tq;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) {
      *reinterpret_cast<float2*>(at + i * 128) = make_float2(o[i][0] * f[0], o[i][1] * f[1]);
      *reinterpret_cast<float2*>(at + i * 128 + 64) = make_float2(o[i][2] * f[0], o[i][3] * f[1]);
    }
  }
};

// Columns 4 c .. of row r of (sequence, head): a / Z, zeros for a row that sees nothing; a NaN stays one.
template <int DH>
__device__ __forceinline__ void p8_write(const PagedAttn& P, int b, int h, int r, int c, float Z, float4 a) {
  const float inv = Z == 0.f ? 0.f : 1.f / Z;
  if (Z == 0.f) a = make_float4(0.f, 0.f, 0.f, 0.f);
  const int i = r / P.group;
  store4((bf16*)P.out + (((size_t)b * P.n + i) * P.hq + h * P.group + (r - i * P.group)) * DH + c * 4, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
}

template <int DH>
__global__ void __launch_bounds__(PG_THREADS, 2) paged8_rows_kernel(const Paged8 PP) {
  using C = P8Cfg<DH>;
  const PagedAttn& P = PP.a;
  pdl_trigger();
  extern __shared__ __align__(128) uint8_t pg_smem[];
  __shared__ PagedLine L;
  __shared__ float sml[PG_WARPS][PG_ROWS][2];
  __shared__ int s_last[2], s_join[2][6];
  __shared__ int s_abort;
  __shared__ __align__(8) unsigned long long bars[PG_WARPS][P8_STAGES];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const scratch = pg_smem + PG_WARPS * P8_STAGES * C::REC + warp * C::SCRATCH;
  uint8_t* const ring = pg_smem + warp * P8_STAGES * C::REC;
  const uint32_t ring_s = smem_u32(ring), bar_s = smem_u32(&bars[warp][0]);
  if (threadIdx.x < PG_WARPS * P8_STAGES) mbar_init(smem_u32(&bars[0][0]) + 8u * threadIdx.x, 1);
  if (threadIdx.x == 0) {
    s_abort = 0;
    s_last[0] = s_last[1] = 0;
  }
  asm volatile("fence.mbarrier_init.release.cluster;\n\tfence.proxy.async.shared::cta;" ::: "memory");
  pdl_wait(KID_ATTN);
  paged_line<true>(L, P, PG_WARPS * P8_BLOCK);          // ends with a barrier
  const int x_begin = L.x_begin, x_end = L.x_end;
  if (x_begin == x_end) return;
  asm volatile("fence.proxy.async.global;" ::: "memory");            // records that earlier kernels' stores wrote are read by copies
  const int R = P.n * P.group;
  const int cap = (int)P.c.cap();

  // ---- copies: the next closed block of this warp ----
  const int per = P.c.shift - 4;
  PagedPlace F = L.first;
  int f_x = x_begin, f_blk = min(L.len[F.b], cap) >> 4;              // closed blocks of F's sequence
  const int* f_table = P.c.table + (size_t)F.b * P.c.max_pages;
  unsigned live = 0u;                        // bit per stage: a copy is under way (not, where the table does not have the block)
  int next = -1, page = -1;                  // the next block, its page
  bool more = false;
  const uint8_t* from = nullptr;             // block 0 of its page 0, its head
  const uint8_t* f_head = PP.pages + (long long)(F.h << per) * C::REC;
  auto look = [&]() {                        // finds the next closed block, a step ahead of its copy
    more = false;
    while (f_x < x_end && !more) {
      next = F.t * PG_WARPS + warp;
      if (next < f_blk) {
        page = f_table[next >> per];
        from = f_head;
        more = true;
      }
      ++f_x;
      if (++F.t == F.T_b && f_x < x_end) {
        F.at(L, P, f_x);
        f_blk = min(L.len[F.b], cap) >> 4;
        f_table = P.c.table + (size_t)F.b * P.c.max_pages;
        f_head = PP.pages + (long long)(F.h << per) * C::REC;
      }
    }
  };
  auto issue = [&](int st) {
    if (!more) return;
    if (page >= 0 && page < P.c.n_pages) {
      live |= 1u << st;
      if (lane == 0) {
        mbar_expect_tx(bar_s + 8u * st, C::REC);
        bulk_load(ring_s + st * C::REC, from + page * PP.page_bytes + (long long)((next & ((1 << per) - 1)) * C::REC), C::REC, bar_s + 8u * st);
      }
    }
    look();
  };
  look();
#pragma unroll
  for (int st = 0; st < P8_STAGES; ++st) issue(st);
  int st = 0;
  unsigned phase = 0u;                       // bit per stage
  bool dead = false;                         // a wait ran out
  Paged8Warp<DH> W;
  PagedPlace S = L.first;
  for (int x = x_begin; x < x_end;) {
    if (x != x_begin) S.at(L, P, x);
    const int b = S.b, h = S.h, mt = S.mt, t0 = S.t, t1 = min(S.T_b, t0 + (x_end - x));
    const int x0 = x - t0;                                           // the item's first tile on the line
    const int len = min(L.len[b], cap), keys = min(len + P.n_new, cap), shut = len >> 4;
    W.begin(P, b, h, mt);
    const bool whole = t0 == 0 && t1 == S.T_b;
    const int place = x == x_begin ? 0 : 1;
    if (!whole && lane == 0 && (warp == 2 || warp == 5)) {           // (while the first copies are on their way)
      int* j = s_join[place];
      if (warp == 2) {
        j[0] = x0; j[1] = b; j[2] = h; j[3] = mt;
        j[4] = place ? (int)blockIdx.x : line_owner(L, x0);
      } else {
        j[5] = line_owner(L, x0 + S.T_b - 1);
      }
    }
    // the open slots first, at most five blocks and so one of this warp: their loads' latency passes while the copies fly
    {
      const int t = max(0, (shut - warp + PG_WARPS - 1) / PG_WARPS), s0 = (t * PG_WARPS + warp) * P8_BLOCK;
      if (t >= t0 && t < t1 && s0 < keys) W.open(PP, b, h, mt, s0, len, keys, any_word(P, b), P.k_new && mt == 0, scratch);
    }
    for (int t = t0; t < t1 && t * PG_WARPS + warp < shut; ++t) {
      if (dead) continue;
      if ((live >> st) & 1u) {
        dead = !__all_sync(0xffffffffu, mbar_wait(bar_s + 8u * st, (phase >> st) & 1u, &s_abort));
        if (dead) continue;
        W.block(P, ring + st * C::REC);
        phase ^= 1u << st;
        live &= ~(1u << st);
      }
      __syncwarp();
      issue(st);
      st = st + 1 == P8_STAGES ? 0 : st + 1;
    }
    // ---- merge of the warps: a thread takes four columns of a row. (Code that runs once per item comes cold from memory, so loops here
    // stay loops.) ----
    const int rows = min(PG_ROWS, R - mt * PG_ROWS), xn = x + (t1 - t0);
    W.finish(reinterpret_cast<float*>(scratch), &sml[warp][0][0]);
    if (dead && lane < PG_ROWS) sml[warp][lane][1] = __int_as_float(0x7fffffff);
    __syncthreads();
    const size_t piece0 = (size_t)blockIdx.x * 2 + place;
    const int mr = threadIdx.x & 7, mc = threadIdx.x >> 3;           // row, columns 4 mc ...
    if (mr < rows && mc < DH / 4) {
      const float* so = reinterpret_cast<const float*>(pg_smem + PG_WARPS * P8_STAGES * C::REC) + mc * 32 + mr;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < PG_WARPS; ++w) M = fmaxf(M, sml[w][mr][0]);
      const float ref = M == -INFINITY ? 0.f : M;
      float Z = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int w = 0; w < PG_WARPS; ++w) {
        const float f = ex2_approx((sml[w][mr][0] - ref) * P.scale_log2);
        const float* y = so + w * (C::SCRATCH / 4);
        Z = fmaf(f, sml[w][mr][1], Z);
        a.x = fmaf(f, y[0], a.x); a.y = fmaf(f, y[8], a.y); a.z = fmaf(f, y[16], a.z); a.w = fmaf(f, y[24], a.w);
      }
      if (whole) {
        p8_write<DH>(P, b, h, mt * PG_ROWS + mr, mc, Z, a);
      } else {
        __stcg(reinterpret_cast<float4*>(P.part_o) + (piece0 * (DH / 4) + mc) * PG_ROWS + mr, a);
        if (mc == 0) __stcg(reinterpret_cast<float2*>(P.part_ml) + piece0 * PG_ROWS + mr, make_float2(M, Z));
      }
    }
    __syncthreads();                                                 // the merge is read before the scratch is written again
    if (!whole && threadIdx.x == 0) {
      // Who delivers the last piece joins them. The count releases this CTA's stores, which came before the barrier, and acquires the others'
      // for the whole CTA, behind the next one.
      const int c0 = s_join[place][4], c1 = s_join[place][5];
      int before;
      asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(P.arrived + c0) : "memory");
      s_last[place] = before == c1 - c0;
    }
    x = xn;
  }
  if (dead) {                                // given up: the copies under way still land before the CTA ends
    const long long t_end = clock64() + WS_WAIT_CYCLES;
    for (int s = 0; s < P8_STAGES; ++s)
      while (((live >> s) & 1u) && !mbar_test(bar_s + 8u * s, (phase >> s) & 1u) && clock64() < t_end) {}
  }

  // ---- join: pieces in the order of their positions, four columns of a row per thread, and as many threads for those as there are ----
  __syncthreads();
#pragma unroll 1
  for (int place = 0; place < 2; ++place) {
    if (!s_last[place]) continue;                                    // the same for the whole CTA
    const int x0 = s_join[place][0], b = s_join[place][1], h = s_join[place][2], mt = s_join[place][3], c0 = s_join[place][4], c1 = s_join[place][5];
    if (threadIdx.x == 0) P.arrived[c0] = 0;                         // as the next call expects it
    const int rows = min(PG_ROWS, R - mt * PG_ROWS), np = c1 - c0 + 1, fp = first_place(L, c0, x0);
    int shift = 3;                                                   // rows as a power of two
    while (shift > 0 && (1 << (shift - 1)) >= rows) --shift;
    const int units = (DH / 4) << shift, subs = PG_THREADS / units, each = (np + subs - 1) / subs;
    const int sub = threadIdx.x / units, unit = threadIdx.x - sub * units, r = unit & ((1 << shift) - 1), c = unit >> shift;
    constexpr int JOIN = 8;                  // pieces under way
    float M = -INFINITY, Z = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float m, float z, const float4& o, float ref) {
      const float f = ex2_approx((m - ref) * P.scale_log2);
      Z = fmaf(f, z, Z);
      a.x = fmaf(f, o.x, a.x); a.y = fmaf(f, o.y, a.y); a.z = fmaf(f, o.z, a.z); a.w = fmaf(f, o.w, a.w);
    };
    auto move = [&](float mx) {                                      // to a new reference
      const float g = ex2_approx((M - (mx == -INFINITY ? 0.f : mx)) * P.scale_log2);
      Z *= g;
      a.x *= g; a.y *= g; a.z *= g; a.w *= g;
      M = mx;
    };
    const float4* po = reinterpret_cast<const float4*>(P.part_o) + c * PG_ROWS + r;
    const float2* pm = reinterpret_cast<const float2*>(P.part_ml) + r;
    const int end = min(np, (sub + 1) * each);
#pragma unroll 1
    for (int i = sub * each; i < end; i += JOIN) {
      float2 ml[JOIN];
      float4 o[JOIN];
#pragma unroll
      for (int u = 0; u < JOIN; ++u) {
        const int k = min(i + u, end - 1), piece = (c0 + k) * 2 + (k == 0 ? fp : 0);
        ml[u] = __ldcg(pm + (size_t)piece * PG_ROWS);
        o[u] = __ldcg(po + (size_t)piece * (DH / 4) * PG_ROWS);
      }
      float mx = M;
#pragma unroll
      for (int u = 0; u < JOIN; ++u) mx = fmaxf(mx, ml[u].x);
      move(mx);
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int u = 0; u < JOIN; ++u)
        if (i + u < end) add(ml[u].x, ml[u].y, o[u], ref);
    }
    if (subs > 1) {
      float* t = reinterpret_cast<float*>(pg_smem) + threadIdx.x;    // [6][256]; the rings are empty
      t[0] = M; t[256] = Z; t[512] = a.x; t[768] = a.y; t[1024] = a.z; t[1280] = a.w;
      __syncthreads();
      if (sub == 0) {
        float mx = M;
        for (int k = 1; k < subs; ++k) mx = fmaxf(mx, t[k * units]);
        move(mx);
        const float ref = mx == -INFINITY ? 0.f : mx;
        for (int k = 1; k < subs; ++k) {
          const float* y = t + k * units;
          add(y[0], y[256], make_float4(y[512], y[768], y[1024], y[1280]), ref);
        }
      }
      __syncthreads();
    }
    if (sub == 0 && r < rows) p8_write<DH>(P, b, h, mt * PG_ROWS + r, c, Z, a);
  }
}

}  // namespace moa
