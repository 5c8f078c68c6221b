// Eviction from a paged key / value cache by accumulated attention weight (sm_100a).
//
// Per (sequence, head) with L slots in use and a budget m < L, the m slots to keep are: the first positions (pos < sink), the
// latest ones (pos >= seen - recent), and of the others those with the largest weight, a NaN after every number, equal weights
// by the lower slot. Keys carry their rotation, so the order of the slots is free: the kept slots behind the budget move into
// the freed slots before it, both in rising order -- at most min(m, L - m) rows move, and no row is both read and written.
//
// What bounds it: the rows that move (4 * dh elements of traffic each), and for small caches the two launches.
//   evict_select_kernel  one CTA per (sequence, head): exact radix selection on 32-bit keys in four passes of 8 bits, then one
//                        ordered pass that lists sources and destinations
//   evict_move_kernel    a warp per moved row, over the whole GPU
#pragma once
#include "moa_paged.cuh"

namespace moa {

constexpr int EV_THREADS = 512;
constexpr int EV_WARPS = EV_THREADS / 32;
constexpr int EV_KEYS = 12288;               // keys kept in shared memory; longer heads read weights and positions again

struct EvictArgs {
  PagedView c;
  int budget, sink, recent;
  int *n_move, *src, *dst;                   // [batch * hkv], [batch * hkv, list_ld]
  int list_ld;
  float* weight_out;
  int* pos_out;
  int* len_out;                              // or null
};

// Rises with the weight; NaN lowest, -0 as +0, protected positions above everything.
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sink, int edge) {
  if (pos < sink || pos >= edge) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictArgs A) {
  pdl_trigger();
  extern __shared__ uint32_t ev_keys[];
  __shared__ int hist[EV_WARPS][256];
  __shared__ int s_bin, s_need, s_cnt[EV_WARPS][3];
  const int bh = blockIdx.x, b = bh / A.c.hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const long long cap = A.c.cap();
  const int L = (int)min((long long)A.c.len[b], cap);
  const int m = A.budget;
  const float* wt = A.c.weight + (size_t)bh * cap;
  const int* ps = A.c.pos + (size_t)bh * cap;
  float* wo = A.weight_out + (size_t)bh * cap;
  int* po = A.pos_out + (size_t)bh * cap;
  const bool apart = wo != wt || po != ps;   // outputs of their own: the slots that stay where they are go there too
  if (L <= m) {
    if (tid == 0) A.n_move[bh] = 0;
    if (apart)
      for (int i = tid; i < L; i += EV_THREADS) { wo[i] = wt[i]; po[i] = ps[i]; }
    return;
  }
  const int edge = (int)max(-2147483648ll, (long long)A.c.seen[b] - A.recent);
  const bool held = L <= EV_KEYS;
  if (held) {
    for (int i = tid; i < L; i += EV_THREADS) ev_keys[i] = evict_key(wt[i], ps[i], A.sink, edge);
    __syncthreads();
  }
  auto key_of = [&](int i) { return held ? ev_keys[i] : evict_key(wt[i], ps[i], A.sink, edge); };
  // the key of rank m (counted from the largest) by four passes of 8 bits
  uint32_t prefix = 0u;
  int need = m;                              // how many of the keys that share the prefix are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < EV_WARPS * 256; i += EV_THREADS) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (int i = tid; i < L; i += EV_THREADS) {
      const uint32_t k = key_of(i);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[warp][(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (tid < 256) {
      int t = 0;
      for (int w = 0; w < EV_WARPS; ++w) t += hist[w][tid];
      hist[0][tid] = t;
    }
    __syncthreads();
    if (warp == 0) {                         // from the top bin down: lane 0 holds bins 255..248, and so on
      int own[8], sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) { own[e] = hist[0][255 - (lane * 8 + e)]; sum += own[e]; }
      int inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      int above = inc - sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (above < need && above + own[e] >= need) { s_bin = 255 - (lane * 8 + e); s_need = need - above; }
        above += own[e];
      }
    }
    __syncthreads();
    prefix |= (uint32_t)s_bin << shift;
    need = s_need;
  }
  // one pass in slot order: of the keys equal to `prefix` the first `need` are kept
  int eq_base = 0, n_src = 0, n_dst = 0;
  int* src = A.src + (size_t)bh * A.list_ld;
  int* dst = A.dst + (size_t)bh * A.list_ld;
  for (int i0 = 0; i0 < L; i0 += EV_THREADS) {
    const int i = i0 + tid;
    const bool in = i < L;
    const uint32_t k = in ? key_of(i) : 0u;
    const bool eq = in && k == prefix;
    const unsigned me = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) s_cnt[warp][0] = __popc(me);
    __syncthreads();
    int before = eq_base, all = 0;
    for (int w = 0; w < EV_WARPS; ++w) { const int c = s_cnt[w][0]; if (w < warp) before += c; all += c; }
    before += __popc(me & ((1u << lane) - 1u));
    eq_base += all;
    const bool keep = in && (k > prefix || (eq && before < need));
    const bool is_src = keep && i >= m, is_dst = in && !keep && i < m;
    const unsigned ms = __ballot_sync(0xffffffffu, is_src), md = __ballot_sync(0xffffffffu, is_dst);
    if (lane == 0) { s_cnt[warp][1] = __popc(ms); s_cnt[warp][2] = __popc(md); }
    __syncthreads();
    int bs = n_src, bd = n_dst;
    for (int w = 0; w < EV_WARPS; ++w) {
      const int cs = s_cnt[w][1], cd = s_cnt[w][2];
      if (w < warp) { bs += cs; bd += cd; }
      n_src += cs;
      n_dst += cd;
    }
    if (apart && keep && i < m) { wo[i] = wt[i]; po[i] = ps[i]; }
    if (is_src) src[bs + __popc(ms & ((1u << lane) - 1u))] = i;
    if (is_dst) dst[bd + __popc(md & ((1u << lane) - 1u))] = i;
    __syncthreads();
  }
  if (tid == 0) A.n_move[bh] = n_src;        // = n_dst: m slots are kept in all
}

// Moves the listed rows with their weights and positions, and writes the new lengths.
template <typename T, int DH>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs A, int per_bh) {
  pdl_trigger();
  pdl_wait();
  const int bh = blockIdx.x / per_bh, part = blockIdx.x - bh * per_bh;
  const int b = bh / A.c.hkv, h = bh - b * A.c.hkv;
  const long long cap = A.c.cap();
  const int n = A.n_move[bh], lane = threadIdx.x & 31;
  const size_t base = (size_t)bh * cap;
  constexpr int CH = DH * (int)sizeof(T) / 16;               // 16-byte pieces per row
  constexpr int PER = 32 / CH > 0 ? 32 / CH : 1;             // rows per warp step
  const int warps = per_bh * 8;
  for (int i0 = (part * 8 + (int)(threadIdx.x >> 5)) * PER; i0 < n; i0 += warps * PER) {
    const int i = i0 + lane / CH, c = lane % CH;
    if (i >= n) continue;
    const int s = A.src[(size_t)bh * A.list_ld + i], d = A.dst[(size_t)bh * A.list_ld + i];
    const long long os = A.c.row(b, s, DH), od = A.c.row(b, d, DH);
    if (os >= 0 && od >= 0) {
      const long long x = (long long)h * DH + c * (16 / (int)sizeof(T));
      const uint4 kv = *reinterpret_cast<const uint4*>((const T*)A.c.k + os + x), vv = *reinterpret_cast<const uint4*>((const T*)A.c.v + os + x);
      *reinterpret_cast<uint4*>((T*)A.c.k + od + x) = kv;
      *reinterpret_cast<uint4*>((T*)A.c.v + od + x) = vv;
    }
    if (c == 0) { A.weight_out[base + d] = A.c.weight[base + s]; A.pos_out[base + d] = A.c.pos[base + s]; }
  }
  if (A.len_out && h == 0 && part == 0 && threadIdx.x == 0) A.len_out[b] = min(A.c.len[b], A.budget);   // len_out may be len
}

}  // namespace moa
