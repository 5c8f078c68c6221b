// Norm of each query and key head, rotation by the row's position, and the store to where the attention reads them, in one pass
// (sm_100a):
//
//   y = x / sqrt(mean x^2 + eps) * gain,  (a, b) -> (a cos - b sin, b cos + a sin) for each pair, angle = position * frequency
//
// What bounds it: every row is read and written once for a few operations per element, so HBM does for prompts, a chain of loads
// for a few rows. A head lies over head_dim / 8 lanes, 16 bytes (bf16) each; its sum of squares and the other half of its pairs
// come by shuffles, so that no shared memory and no barrier is in the way. Normalising is linear, so gain, cosine and sine are
// multiplied once per row: an element costs one product with itself and one with its partner, and one with the root.
// A warp takes a row and a number of its heads: all of a kind's when there are many rows, so that the row's angles are formed
// once for them; eight or sixteen when there are few, so that the heads spread over the GPU.
// Angles: position * frequency in 64 bits, reduced to a fraction of a turn there (a position of 100000 leaves fp32 no more than
// 7 bits behind the turn), then cosine and sine in fp32. A warp's lanes form two each and pass them round.
// Measured: 32768 rows of 48 heads of 128 (0.81 GB read and written, values too) 201 us = 4.0 TB/s; 1024 rows of 80 heads 15.0 us.
#pragma once
#include "moa_paged.cuh"

namespace moa {

constexpr int QN_WARPS = 8;
constexpr int QN_U = 4;                      // heads per lane under way

struct QkNormArgs {
  const void *q, *k, *v;                     // rows q_stride / kv_stride elements apart; v null: not copied
  void *q_out, *k_out;                       // rows of hq * DH and hkv * DH; k_out null: to the pages
  long long q_stride, kv_stride, q_out_stride, k_out_stride;
  const void *q_gain, *k_gain;               // [DH] or null: no norm for either
  const int* pos;                            // [rows], < 0: padding
  const double* freq;                        // [rot / 2], radians per position
  const long long* slot;                     // [rows], with pages
  void *pk, *pv;
  long long page_stride, n_slots;            // n_pages << shift
  int shift, rows, hq, hkv, rot, inter;
  int per;                                   // heads of a unit of work
  int uq, ukv;                               // units of a row: of its queries, of its keys (or values)
  float eps;
};

template <typename T> struct Raw8;           // eight neighbouring elements of a row
template <> struct Raw8<bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = __ldcg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void store(bf16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void get(float* x) const { bf16x8_to_float(w, x); }
  __device__ __forceinline__ void set(const float* x) {
    w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
  __device__ __forceinline__ Raw8 from(int lane) const {
    Raw8 r;
    r.w.x = __shfl_sync(0xffffffffu, w.x, lane); r.w.y = __shfl_sync(0xffffffffu, w.y, lane);
    r.w.z = __shfl_sync(0xffffffffu, w.z, lane); r.w.w = __shfl_sync(0xffffffffu, w.w, lane);
    return r;
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = __ldcg(reinterpret_cast<const float4*>(p)); b = __ldcg(reinterpret_cast<const float4*>(p) + 1); }
  __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = a; reinterpret_cast<float4*>(p)[1] = b; }
  __device__ __forceinline__ void get(float* x) const { x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w; }
  __device__ __forceinline__ void set(const float* x) { a = make_float4(x[0], x[1], x[2], x[3]); b = make_float4(x[4], x[5], x[6], x[7]); }
  __device__ __forceinline__ Raw8 from(int lane) const {
    Raw8 r;
    r.a.x = __shfl_sync(0xffffffffu, a.x, lane); r.a.y = __shfl_sync(0xffffffffu, a.y, lane);
    r.a.z = __shfl_sync(0xffffffffu, a.z, lane); r.a.w = __shfl_sync(0xffffffffu, a.w, lane);
    r.b.x = __shfl_sync(0xffffffffu, b.x, lane); r.b.y = __shfl_sync(0xffffffffu, b.y, lane);
    r.b.z = __shfl_sync(0xffffffffu, b.z, lane); r.b.w = __shfl_sync(0xffffffffu, b.w, lane);
    return r;
  }
};

template <typename T, int DH>
__global__ void __launch_bounds__(QN_WARPS * 32) qk_norm_rope_kernel(const QkNormArgs A) {
  constexpr int LPH = DH / 8, HP = 32 / LPH;                         // lanes per head, heads side by side in a warp
  pdl_trigger();
  pdl_wait(KID_ROPE);
  const int lane = threadIdx.x & 31, li = lane % LPH, sub = lane / LPH;
  const int units = A.uq + (A.v ? 2 : 1) * A.ukv;
  const long long w = (long long)blockIdx.x * QN_WARPS + (threadIdx.x >> 5);
  const long long row = w / units;
  if (row >= A.rows) return;
  const int u = (int)(w - row * units);
  const int kind = u < A.uq ? 0 : u < A.uq + A.ukv ? 1 : 2;          // queries, keys, values
  const int h0 = (kind == 0 ? u : (u - A.uq) % A.ukv) * A.per, h1 = min(h0 + A.per, kind == 0 ? A.hq : A.hkv);
  const int pos = A.pos[row];
  if (pos < 0) return;
  const T* src = (const T*)(kind == 0 ? A.q : kind == 1 ? A.k : A.v) + row * (kind == 0 ? A.q_stride : A.kv_stride);
  T* dst;
  if (kind == 0) {
    dst = (T*)A.q_out + row * A.q_out_stride;
  } else if (A.k_out) {
    dst = (T*)A.k_out + row * A.k_out_stride;
  } else {
    const long long s = A.slot[row];
    if (s < 0 || s >= A.n_slots) return;
    dst = (T*)(kind == 1 ? A.pk : A.pv) + (s >> A.shift) * A.page_stride + (s & ((1ll << A.shift) - 1)) * (long long)A.hkv * DH;
  }
  Raw8<T> x[QN_U];
  auto fetch = [&](int h) {
#pragma unroll
    for (int i = 0; i < QN_U; ++i) x[i].load(src + (long long)min(h + i * HP + sub, h1 - 1) * DH + li * 8);      // behind the last head: that one
  };
  fetch(h0);
  if (kind == 2) {
    for (int h = h0; h < h1; h += QN_U * HP) {
      if (h != h0) fetch(h);
#pragma unroll
      for (int i = 0; i < QN_U; ++i)
        if (h + i * HP + sub < h1) x[i].store(dst + (long long)(h + i * HP + sub) * DH + li * 8);
    }
    return;
  }
  // ---- factors of this lane's elements and of their partners ----
  const int half = A.rot >> 1;
  float c2[2], s2[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    c2[e] = 1.f;
    s2[e] = 0.f;
    if (lane + 32 * e < half) {
      const double t = (double)pos * A.freq[lane + 32 * e] * 0.15915494309189533577;
      sincospif(2.f * (float)(t - rint(t)), &s2[e], &c2[e]);
    }
  }
  const T* gain = (const T*)(kind == 0 ? A.q_gain : A.k_gain);
  int partner = lane;                        // lane that has the other elements of this lane's pairs
  float g[8], gp[8], own[8], other[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = gp[e] = 1.f;
  const bool turns = li * 8 < A.rot, low = li * 8 < half;
  if (!A.inter && turns) partner = low ? lane + (half >> 3) : lane - (half >> 3);
  if (gain) {
    Raw8<T> t;
    t.load(gain + li * 8);
    t.get(g);
    t.load(gain + (li + partner - lane) * 8);
    t.get(gp);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int f = A.inter ? li * 4 + (e >> 1) : (low ? li : li - (half >> 3)) * 8 + e;       // its frequency; out of range where nothing turns
    const float ca = __shfl_sync(0xffffffffu, c2[0], f & 31), cb = __shfl_sync(0xffffffffu, c2[1], f & 31);
    const float sa = __shfl_sync(0xffffffffu, s2[0], f & 31), sb = __shfl_sync(0xffffffffu, s2[1], f & 31);
    const float c = !turns ? 1.f : f & 32 ? cb : ca, s = !turns ? 0.f : f & 32 ? sb : sa;
    const bool first = A.inter ? (e & 1) == 0 : low;                 // the pair's first element
    own[e] = g[e] * c;
    other[e] = (A.inter ? g[e ^ 1] : gp[e]) * (first ? -s : s);
  }
  for (int h = h0; h < h1; h += QN_U * HP) {
    if (h != h0) fetch(h);
#pragma unroll
    for (int i = 0; i < QN_U; ++i) {
      float a[8], b[8];
      x[i].get(a);
      float root = 1.f;
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(a[e], a[e], ss);
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        root = rsqrtf(ss * (1.f / DH) + A.eps);
      }
      if (A.inter) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = a[e ^ 1];
      } else {
        x[i].from(partner).get(b);
      }
      // an element that does not turn takes no part of a partner, whatever that is
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = root * (turns ? fmaf(other[e], b[e], own[e] * a[e]) : own[e] * a[e]);
      x[i].set(a);
      if (h + i * HP + sub < h1) x[i].store(dst + (long long)(h + i * HP + sub) * DH + li * 8);
    }
  }
}

}  // namespace moa
