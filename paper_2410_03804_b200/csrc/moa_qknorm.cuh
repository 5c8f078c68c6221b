// Norm of each query and key head, rotation by the row's position, and the store to where the attention reads them, in one pass
// (sm_100a):
//
//   y = x / sqrt(mean x^2 + eps) * gain,  (a, b) -> (a cos - b sin, b cos + a sin) for each pair, angle = position * frequency
//
// What bounds it: every row is read and written once for a few operations per element, so HBM does for prompts, a chain of loads
// for a few rows. A head lies over head_dim / 8 lanes, 16 bytes (bf16) each; its sum of squares and the other half of its pairs
// come by shuffles, so that no shared memory and no barrier is in the way. Normalising is linear, so gain, cosine and sine are
// multiplied once per row: an element costs one product with itself and one with its partner, and one with the root.
// Work is cut into groups of heads of one kind of one row, what a warp has under way at once, and the warps take equal consecutive
// stretches of them, the next group's loads out before the last one is worked on. So the row's angles are formed once for all that a
// stretch holds of it, and one group per warp spreads the heads of a few rows over the GPU. (A warp per row and kind, without
// the loads ahead: 197 us for the large case below, 14 of 24 warps of an SM there on average.)
// Angles: position * frequency in 64 bits, reduced to a fraction of a turn there (a position of 100000 leaves fp32 no more than
// 7 bits behind the turn), then cosine and sine in fp32. A warp's lanes form two each and pass them round.
// Measured, calls in a graph: 32768 rows of 32 + 2 x 8 heads of 128, bf16 (0.81 GB): 144 us, 5.6 TB/s, 0.85 of a copy's; 16 x 61 rows of
// 64 + 2 x 8 heads (40 MB, which L2 holds): 11.0 us; 33 rows of 4 + 4 heads of 64, fp32: 3.0 us, the chain of loads and a launch.
#pragma once
#include "moa_paged_tc.cuh"

namespace moa {

constexpr int QN_WARPS = 4;
constexpr int QN_U = 4;                      // heads per lane under way
constexpr int QN_RESIDENT = 4;               // CTAs per SM

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
  int gq, gkv;                               // groups of a row: of its queries, of its keys (or values)
  int span;                                  // groups that a warp takes
  float eps;
};

// Eight neighbouring elements of a row. Rows pass once, so they are marked to leave L2 first (155 to 149 us for the large case below).
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_kept(const bf16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(bf16* p) const { __stcs(reinterpret_cast<uint4*>(p), w); }
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
  __device__ __forceinline__ void load(const float* p) { a = __ldcs(reinterpret_cast<const float4*>(p)); b = __ldcs(reinterpret_cast<const float4*>(p) + 1); }
  __device__ __forceinline__ void load_kept(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void store(float* p) const { __stcs(reinterpret_cast<float4*>(p), a); __stcs(reinterpret_cast<float4*>(p) + 1, b); }
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

__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// FULL: every element turns.
template <typename T, int DH, bool FULL>
__global__ void __launch_bounds__(QN_WARPS * 32, QN_RESIDENT) qk_norm_rope_kernel(const QkNormArgs A) {
  constexpr int LPH = DH / 8, HP = 32 / LPH;                         // lanes per head, heads side by side in a warp
  pdl_trigger();
  pdl_wait(KID_ROPE);
  const int lane = threadIdx.x & 31, li = lane % LPH, sub = lane / LPH;
  const int G = A.gq + (A.v ? 2 : 1) * A.gkv;                        // groups of a row
  const long long total = (long long)A.rows * G;
  long long g = ((long long)blockIdx.x * QN_WARPS + (threadIdx.x >> 5)) * A.span;
  if (g >= total) return;
  const long long g_end = min(g + A.span, total);
  int row = (int)(g / G), u = (int)(g - (long long)row * G);
  const int half = A.rot >> 1;
  const bool turns = FULL || li * 8 < A.rot, low = li * 8 < half;
  const int partner = A.inter || !turns ? lane : low ? lane + (half >> 3) : lane - (half >> 3);       // the lane with the other elements of this lane's pairs

  Raw8<T> x[QN_U], y[QN_U];
  auto kind_of = [&](int v) { return v < A.gq ? 0 : v < A.gq + A.gkv ? 1 : 2; };                      // queries, keys, values
  auto fetch = [&](Raw8<T>* z, int r, int v) {
    const int kind = kind_of(v), h0 = (v - (kind == 0 ? 0 : kind == 1 ? A.gq : A.gq + A.gkv)) * (QN_U * HP), last = (kind == 0 ? A.hq : A.hkv) - 1;
    const T* src = (const T*)(kind == 0 ? A.q : kind == 1 ? A.k : A.v) + r * (kind == 0 ? A.q_stride : A.kv_stride) + li * 8;
#pragma unroll
    for (int i = 0; i < QN_U; ++i) z[i].load(src + (long long)min(h0 + i * HP + sub, last) * DH);     // behind the last head: that one
  };
  fetch(x, row, u);
  int kind_now = -1, row_now = -1, pos = -1;
  long long slot = -1;
  float c2[2], s2[2];                        // cosine and sine of pairs lane and lane + 32
  uint64_t own[4], other[4];                 // factors of this lane's elements and of their partners, two at a time
#pragma unroll 1
  for (; g < g_end; ++g) {
    const int r = row, v = u, kind = kind_of(v);
    if (++u == G) { u = 0; ++row; }
    if (g + 1 < g_end) fetch(y, row, u);
    if (r != row_now) {
      row_now = r;
      kind_now = -1;
      pos = A.pos[r];
      slot = 0;
      if (!A.k_out) {
        slot = A.slot[r];
        if (slot >= A.n_slots) slot = -1;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        c2[e] = 1.f;
        s2[e] = 0.f;
        if (lane + 32 * e < half) {
          const double t = (double)pos * A.freq[lane + 32 * e] * 0.15915494309189533577;
          sincospif(2.f * (float)(t - rint(t)), &s2[e], &c2[e]);
        }
      }
    }
    const T* gain = (const T*)(kind == 0 ? A.q_gain : A.k_gain);
    if (pos >= 0 && kind != 2 && kind != kind_now) {
      kind_now = kind;
      float w[8], wp[8], o[8], p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = wp[e] = 1.f;
      if (gain) {
        Raw8<T> t;
        t.load_kept(gain + li * 8);
        t.get(w);
        t.load_kept(gain + (li + partner - lane) * 8);
        t.get(wp);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int f = A.inter ? li * 4 + (e >> 1) : (low ? li : li - (half >> 3)) * 8 + e;            // its frequency; out of range where nothing turns
        const float ca = __shfl_sync(0xffffffffu, c2[0], f & 31), cb = __shfl_sync(0xffffffffu, c2[1], f & 31);
        const float sa = __shfl_sync(0xffffffffu, s2[0], f & 31), sb = __shfl_sync(0xffffffffu, s2[1], f & 31);
        const float c = !turns ? 1.f : f & 32 ? cb : ca, s = !turns ? 0.f : f & 32 ? sb : sa;
        const bool first = A.inter ? (e & 1) == 0 : low;             // the pair's first element
        o[e] = w[e] * c;
        p[e] = (A.inter ? w[e ^ 1] : wp[e]) * (first ? -s : s);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) { own[e] = f2_pack(o[2 * e], o[2 * e + 1]); other[e] = f2_pack(p[2 * e], p[2 * e + 1]); }
    }
    if (pos >= 0 && (kind == 0 || slot >= 0)) {
      const int h0 = (v - (kind == 0 ? 0 : kind == 1 ? A.gq : A.gq + A.gkv)) * (QN_U * HP), heads = kind == 0 ? A.hq : A.hkv;
      T* dst = kind == 0 ? (T*)A.q_out + r * A.q_out_stride
               : A.k_out ? (T*)A.k_out + r * A.k_out_stride
                         : (T*)(kind == 1 ? A.pk : A.pv) + (slot >> A.shift) * A.page_stride + (slot & ((1ll << A.shift) - 1)) * (long long)A.hkv * DH;
      dst += (long long)(h0 + sub) * DH + li * 8;
#pragma unroll
      for (int i = 0; i < QN_U; ++i) {
        if (kind != 2) {
          float a[8], b[8];
          x[i].get(a);
          uint64_t z[4], root2 = f2_pack(1.f, 1.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = f2_pack(a[2 * e], a[2 * e + 1]);
          if (gain) {
            uint64_t ss2 = 0ull;
#pragma unroll
            for (int e = 0; e < 4; ++e) ss2 = f2_fma(z[e], z[e], ss2);
            float ss, st;
            f2_unpack(ss2, ss, st);
            ss += st;
#pragma unroll
            for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float root = rsqrtf(ss * (1.f / DH) + A.eps);
            root2 = f2_pack(root, root);
          }
          if (A.inter) {
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = a[e ^ 1];
          } else {
            x[i].from(partner).get(b);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint64_t w = f2_mul(own[e], z[e]);
            // an element that does not turn takes no part of a partner, whatever that is
            if (FULL || turns) w = f2_fma(other[e], f2_pack(b[2 * e], b[2 * e + 1]), w);
            f2_unpack(f2_mul(w, root2), a[2 * e], a[2 * e + 1]);
          }
          x[i].set(a);
        }
        if (h0 + i * HP + sub < heads) x[i].store(dst + (long long)i * HP * DH);
      }
    }
#pragma unroll
    for (int i = 0; i < QN_U; ++i) x[i] = y[i];
  }
}

}  // namespace moa
