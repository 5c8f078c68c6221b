// The rules that an LLM's logits pass before a token is chosen (sm_100a): penalties for tokens of the context, biases,
// a mask of allowed tokens; and their arg-max, so that a verification needs no adjusted logits in memory.
//
// Context of row (b, i) = the sequence's record (prompt and generated tokens) + the path root .. i of the draft tree. For
// logit x of token t, in fp32 and in this order, each step rounded once:
//   t in the context:     x = x > 0 ? x / repetition : x * repetition
//   c times generated:    x = x - frequency * c;   c > 0: x = x - presence      (c: record's count + occurrences on the path)
//   biases of t:          x = x + (their sum, in list order)
//   t not allowed:        x = -inf
// choice = the smallest token among the largest x before x is rounded to the logits' type; NaN never wins, and a row that
// leaves nothing above -inf chooses token 0.
//
// What bounds it: the logits, streamed once (and written once when adjusted logits are wanted). The rules are sparse: a
// record knows a few thousand of 128256 tokens. A CTA (or eight in a cluster) takes a row. It marks the allowed tokens of its
// slice that any other rule touches (the record's, the path's, the biased ones) in a bitmap in shared memory, lists them, and
// takes the listed ones side by side over its threads, so that their scattered loads (logit, count) are under way together;
// path and biases are in a small hash table. The stream then looks at bits only, in shared memory: a masked or listed token
// counts as -inf, four tokens of a table's byte selectors at a time, and the place of the best of 16 bytes is looked up once,
// at the end. Pieces are loaded four ahead. When a CTA has a row of its own, a quarter of its warps take the list while the
// others stream.
// Measured, 976 rows of 128256 bf16 with 300 biases: 70 us = 3.8 TB/s (73 us when the following were tried), of which the
// bitmap, the table and the list take the first 15 us of a CTA. The allowed bits read again as bytes from global memory beside
// each piece: 109 us; list first, then the stream by all warps: 82 us; listed tokens taken by the stream as it met them: 284 us;
// a CTA walking the rows of a sequence with one list for all: 131 us, its rows' dependent steps no longer hidden by other CTAs.
// CTAs of 128 threads, seven to an SM and all rows at once: 85 us against 73 us of 256 threads.
#pragma once
#include "moa_verify.cuh"

namespace moa {

constexpr int RU_MAX_PATH = 256;             // tree slots per sequence
constexpr int RU_MAX_BIAS = 1024;
constexpr int RU_THREADS = 256;               // of a CTA that takes a row alone
constexpr int RU_LIST = 1280;                // listed tokens of a slice; those behind them are taken one by one

struct RulesArgs {
  const int* counts;                         // [batch, V] or null
  const unsigned* seen;                      // [batch, words] or null
  const float *rep, *freq, *pres;            // [batch] or null
  const int* bias_id;                        // [batch, n_bias]
  const float* bias_val;
  const unsigned* allow;                     // [batch, n, words] or null
  const int *tok, *parent;                   // [batch, n] or null
  int n_bias, n, V, words, table;            // table: hash slots, a power of two (0: no path and no bias)
  const void* x;                             // T [batch, n, V]
  void* out;                                 // T [batch, n, V] or null; may be x
  int* choice;                               // [batch, n] or null
};

__device__ __forceinline__ unsigned ru_hash(int id, unsigned mask) { return ((unsigned)id * 2654435761u >> 12) & mask; }

// Rises with the value, -0 as +0; 0 for -inf and NaN.
__device__ __forceinline__ unsigned ru_key(float v) {
  if (!(v > -INFINITY)) return 0u;
  const unsigned u = __float_as_uint(v + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <typename T, int CL, int NT>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT) rules_kernel(const RulesArgs A) {
  pdl_trigger();
  extern __shared__ __align__(16) uint32_t ru_smem[];
  __shared__ float cv[CL];
  __shared__ int ci[CL];
  __shared__ int s_path[RU_MAX_PATH];
  __shared__ int s_np, s_listed, s_step;
  __shared__ int list[RU_LIST];                    // before it is filled: tokens and parents of the tree
  int *s_tok = list, *s_par = list + RU_MAX_PATH;
  __shared__ uint2 picks[256];                     // 16-bit types: byte selectors of four words for every byte of mask bits
  __shared__ uint2 best[2][NT / 32];               // per warp: stream (key, first token of its 16 bytes), touched (key, token)
  const int rank = blockIdx.x, row = blockIdx.y, b = row / A.n, ti = row - b * A.n;
  const int tid = threadIdx.x;
  const int per_cta = ((A.V + CL - 1) / CL + 31) & ~31;
  const int e0 = min(A.V, rank * per_cta), e1 = min(A.V, e0 + per_cta);
  const int n_words = (e1 - e0 + 31) >> 5;
  // shared memory: hash table (id; path count + 2^16 * bias entries; lowest of them, later the bias), then the slice's bitmap
  int* h_id = reinterpret_cast<int*>(ru_smem);
  int* h_cnt = h_id + A.table;
  int* h_first = h_cnt + A.table;
  float* h_val = reinterpret_cast<float*>(h_first);
  uint32_t* mark = reinterpret_cast<uint32_t*>(h_first + A.table);
  const unsigned hmask = A.table > 0 ? (unsigned)A.table - 1u : 0u;
  // every CTA of the cluster is running before another writes to its shared memory (waited for at the end)
  if constexpr (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  pdl_wait();

  const int* counts = A.counts ? A.counts + (size_t)b * A.V : nullptr;
  const unsigned* seen = A.seen ? A.seen + (size_t)b * A.words + (e0 >> 5) : nullptr;
  const unsigned* allow = A.allow ? A.allow + (size_t)row * A.words + (e0 >> 5) : nullptr;
  const bool dense = counts && !seen;        // counts without the record's bits: every count is read
  if constexpr (sizeof(T) == 2) {                  // bit 2 q: the low half of word q, bit 2 q + 1: its high half; 0: from the other operand
    auto pick = [](unsigned two) { return 0x7654u - (two & 1u) * 0x0044u - (two >> 1) * 0x4400u; };
    for (int i = tid; i < 256; i += NT) picks[i] = make_uint2(pick(i & 3) | pick((i >> 2) & 3) << 16, pick((i >> 4) & 3) | pick((i >> 6) & 3) << 16);
  }
  if (tid == 0) s_listed = s_step = 0;
  // ---- bitmap and hash table ----
  const int size = e1 - e0;
  auto in_slice = [&](int id) { return id >= e0 && id < e1; };
  auto may = [&](int e) { return !allow || ((allow[e >> 5] >> (e & 31)) & 1u) != 0u; };
  if (dense) {
    for (int i = tid; i < ((size + 31) & ~31); i += NT) {             // whole warps
      const unsigned m = __ballot_sync(0xffffffffu, i < size && counts[e0 + min(i, size - 1)] > 0);
      if ((i & 31) == 0) mark[i >> 5] = allow ? m & allow[i >> 5] : m;
    }
  } else {
    for (int i0 = tid; i0 < n_words; i0 += 4 * NT) {
      unsigned m[4], a[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = min(i0 + u * NT, n_words - 1);
        m[u] = seen ? seen[i] : 0u;
        a[u] = allow && seen ? allow[i] : ~0u;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * NT, left = size - i * 32;              // no bits behind the vocabulary
        if (i < n_words) mark[i] = m[u] & a[u] & (left >= 32 ? ~0u : (1u << left) - 1u);
      }
    }
  }
  if (A.table > 0) {
    for (int i = tid; i < A.table; i += NT) { h_id[i] = -1; h_cnt[i] = 0; h_first[i] = 0x7fffffff; }
    if (A.tok)
      for (int i = tid; i < A.n; i += NT) { s_tok[i] = A.tok[(size_t)b * A.n + i]; s_par[i] = A.parent[(size_t)b * A.n + i]; }
    __syncthreads();
    if (tid == 0) {                          // root .. this slot; an unused slot (parent < 0 behind the root) has no path
      int np = 0;
      if (A.tok && (ti == 0 || s_par[ti] >= 0))
        for (int j = ti; j >= 0;) {
          s_path[np++] = s_tok[j];
          const int p = s_par[j];
          if (j == 0 || p >= j) break;
          j = p;
        }
      s_np = np;
    }
    auto slot_of = [&](int id) {             // the table has at least a third more slots than can be asked for
      unsigned s = ru_hash(id, hmask);
      while (true) {
        const int old = atomicCAS(&h_id[s], -1, id);
        if (old == -1 || old == id) return (int)s;
        s = (s + 1u) & hmask;
      }
    };
    const int* bid = A.bias_id + (size_t)b * A.n_bias;
    const float* bval = A.bias_val + (size_t)b * A.n_bias;
    for (int i = tid; i < A.n_bias; i += NT) {
      const int id = bid[i];
      if (!in_slice(id) || !may(id - e0)) continue;
      const int s = slot_of(id);
      atomicAdd(&h_cnt[s], 1 << 16);
      atomicMin(&h_first[s], i);
      atomicOr(&mark[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    __syncthreads();
    const int np = s_np;
    for (int i = tid; i < np; i += NT) {
      const int id = s_path[i];
      if (!in_slice(id) || !may(id - e0)) continue;
      atomicAdd(&h_cnt[slot_of(id)], 1);
      atomicOr(&mark[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    for (int s = tid; s < A.table; s += NT) {          // (the path only adds entries without a bias)
      const int entries = h_cnt[s] >> 16;
      if (entries == 0) continue;
      const int i0 = h_first[s], id = h_id[s];
      float v = bval[i0];
      if (entries > 1)                        // the same id twice: summed in list order, whatever order the threads came in
        for (int i = i0 + 1; i < A.n_bias; ++i)
          if (bid[i] == id) v = __fadd_rn(v, bval[i]);
      h_val[s] = v;
    }
  }
  __syncthreads();

  // ---- the list of the marked tokens, in no order, and the bits of those that the stream takes: allowed, not marked ----
  const T* xr = (const T*)A.x + (size_t)row * A.V;
  T* orow = A.out ? (T*)A.out + (size_t)row * A.V : nullptr;
  const float rep = A.rep ? A.rep[b] : 1.f, freq = A.freq ? A.freq[b] : 0.f, pres = A.pres ? A.pres[b] : 0.f;
  float tv = -INFINITY;                            // best of the touched tokens
  int te = 0x7fffffff;
  // one touched token of the slice
  auto touch = [&](int e, float x, bool known, int c) {
    bool biased = false;
    float bias = 0.f;
    if (A.table > 0) {
      for (unsigned s = ru_hash(e0 + e, hmask);; s = (s + 1u) & hmask) {
        const int id = h_id[s];
        if (id == -1) break;
        if (id == e0 + e) {
          const int on_path = h_cnt[s] & 0xffff;
          c += on_path;
          known = known || on_path > 0;
          biased = (h_cnt[s] >> 16) > 0;
          bias = h_val[s];
          break;
        }
      }
    }
    known = known || c > 0;
    if (known && A.rep) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
    if (c > 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, (float)c)), pres);
    if (biased) x = __fadd_rn(x, bias);
    if (orow) orow[e0 + e] = from_f<T>(x);
    best_of(x, e, tv, te);
  };
  auto in_record = [&](int e) { return seen && ((seen[e >> 5] >> (e & 31)) & 1u); };
  uint32_t* pass = A.out ? mark + ((per_cta + 31) >> 5) + 1 : mark;      // without an output nobody asks for the marks again
  for (int w0 = tid; w0 < n_words; w0 += 4 * NT) {
    unsigned a[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) a[u] = allow ? allow[min(w0 + u * NT, n_words - 1)] : ~0u;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int wi = w0 + u * NT;
      if (wi >= n_words) break;
      unsigned m = mark[wi];
      pass[wi] = a[u] & ~m;
      if (m == 0u) continue;
      int at = atomicAdd(&s_listed, __popc(m));
      for (; m != 0u; m &= m - 1u, ++at) {
        const int e = wi * 32 + __ffs(m) - 1;
        if (at < RU_LIST) {
          list[at] = e;
        } else {                                   // (rare) no room
          const bool known = in_record(e);
          touch(e, to_f(xr[e0 + e]), known, counts && (known || dense) ? __ldcg(counts + e0 + e) : 0);
        }
      }
    }
  }
  __syncthreads();

  // ---- the stream's first batch sets out, then the listed tokens ----
  constexpr int PER = 16 / sizeof(T), UN = 4;
  constexpr unsigned ALL = (1u << PER) - 1u;
  const uint8_t* mark8 = reinterpret_cast<const uint8_t*>(mark);
  const uint8_t* pass8 = reinterpret_cast<const uint8_t*>(pass);
  // the row's 16-byte pieces start `head` tokens into the slice; with an output that does not lie alike, there are none
  const T* xs = xr + e0;
  T* os = orow ? orow + e0 : nullptr;
  const int head = os && (((uintptr_t)xs ^ (uintptr_t)os) & 15u) ? size : min(size, (int)((16u - (unsigned)((uintptr_t)xs & 15u)) % 16u / sizeof(T)));
  const int nvec = (size - head) / PER, tail = head + nvec * PER;
  uint4 raw[UN];                                   // pieces under way: one that was taken is replaced at once
  auto load = [&](int c, uint4& x) {
    if (c < nvec) x = __ldcs(reinterpret_cast<const uint4*>(xs + head) + c);
  };
  auto bits_of = [&](const uint8_t* bits, int e) -> unsigned {
    unsigned v = bits[e >> 3];
    if ((e & 7) > 8 - PER) v |= (unsigned)bits[(e >> 3) + 1] << 8;
    return v >> (e & 7) & ALL;
  };
  // A row's CTA: a quarter of the warps take the listed tokens while the others stream, and who gets to it takes the next
  // UN * 32 pieces. A slice of eight has a few listed tokens per warp: all warps take them, their first pieces under way.
  constexpr bool SPLIT = CL == 1;
  constexpr int LT = SPLIT ? NT / 4 : NT;
  const int lane = tid & 31, wid = tid >> 5;
  int c0 = wid * UN * 32 + lane;
  auto next_step = [&](int c) {
    if (!SPLIT) return c + UN * NT;
    int step = 0;
    if (lane == 0) step = atomicAdd(&s_step, UN * 32);
    return __shfl_sync(0xffffffffu, step, 0) + lane;
  };
  auto first_step = [&]() {
    if (SPLIT) c0 = next_step(0);
#pragma unroll
    for (int u = 0; u < UN; ++u) load(c0 + u * 32, raw[u]);
  };
  if (!SPLIT || tid >= LT) first_step();
  if (tid < LT) {
    const int n_list = min(s_listed, RU_LIST);
    for (int k0 = tid; k0 < n_list; k0 += 4 * LT) {
      int e[4], c[4];
      float x[4];
      bool known[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        e[u] = k0 + u * LT < n_list ? list[k0 + u * LT] : -1;
        if (e[u] < 0) continue;
        x[u] = to_f(xs[e[u]]);
        known[u] = in_record(e[u]);
        c[u] = counts ? __ldcg(counts + e0 + e[u]) : 0;         // without its bit it does not count
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e[u] >= 0) touch(e[u], x[u], known[u], known[u] || dense ? c[u] : 0);
    }
    // the few tokens before and behind the pieces
    for (int k = tid; k < head + size - tail; k += LT) {
      const int e = k < head ? k : tail + k - head;
      if (os && ((mark8[e >> 3] >> (e & 7)) & 1u)) continue;
      const T x = (pass8[e >> 3] >> (e & 7)) & 1u ? xs[e] : from_f<T>(-INFINITY);
      if (os) os[e] = x;                           // the bits of a NaN included, as the pieces are passed on
      best_of(to_f(x), e, tv, te);
    }
    if (SPLIT) first_step();
  }
  float bv = -INFINITY;                            // best of the stream
  int be = 0x7fffffff;                             // the first token of the 16 bytes it is in
  while (c0 - lane < nvec) {
    const int c1 = next_step(c0);
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int c = c0 + u * 32, e = head + c * PER;
      if (c >= nvec) break;
      const unsigned in = bits_of(pass8, e);
      uint4 w;
      float vm;
      if constexpr (sizeof(T) == 4) {
        w = make_uint4(in & 1u ? raw[u].x : 0xff800000u, in & 2u ? raw[u].y : 0xff800000u, in & 4u ? raw[u].z : 0xff800000u, in & 8u ? raw[u].w : 0xff800000u);
        vm = fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
      } else {
        const uint2 p = picks[in];
        w = make_uint4(__byte_perm(raw[u].x, 0xff80ff80u, p.x), __byte_perm(raw[u].y, 0xff80ff80u, p.x >> 16),
                       __byte_perm(raw[u].z, 0xff80ff80u, p.y), __byte_perm(raw[u].w, 0xff80ff80u, p.y >> 16));
        auto two = [](uint32_t v) { return *reinterpret_cast<__nv_bfloat162*>(&v); };
        const __nv_bfloat162 m = __hmax2(__hmax2(two(w.x), two(w.y)), __hmax2(two(w.z), two(w.w)));       // NaN only of NaNs
        const uint32_t mw = *reinterpret_cast<const uint32_t*>(&m);
        vm = fmaxf(__uint_as_float(mw << 16), __uint_as_float(mw & 0xffff0000u));
      }
      load(c1 + u * 32, raw[u]);
      be = vm > bv ? e : be;                       // rising tokens: the first of equals stays
      bv = fmaxf(bv, vm);
      if (os) {
        const unsigned skip = bits_of(mark8, e);   // marked: written by the list's threads
        if (skip == 0u) {
          __stcs(reinterpret_cast<uint4*>(os + e), w);
        } else {
#pragma unroll
          for (int q = 0; q < PER; ++q)
            if (!((skip >> q) & 1u)) {
              const uint32_t v = sizeof(T) == 4 ? (q == 0 ? w.x : q == 1 ? w.y : q == 2 ? w.z : w.w) : (q < 2 ? w.x : q < 4 ? w.y : q < 6 ? w.z : w.w);
              if constexpr (sizeof(T) == 4) os[e + q] = __uint_as_float(v);
              else os[e + q] = __ushort_as_bfloat16((unsigned short)(v >> (16 * (q & 1))));
            }
        }
      }
    }
    c0 = c1;
  }

  if constexpr (CL > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (!A.choice) return;                           // the same for the whole grid
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const unsigned key = ru_key(kind ? tv : bv);
    const unsigned top = __reduce_max_sync(0xffffffffu, key);
    const unsigned at = __reduce_min_sync(0xffffffffu, key == top ? (unsigned)(kind ? te : be) : 0x7fffffffu);
    if (lane == 0) best[kind][wid] = make_uint2(top, at);
  }
  __syncthreads();
  if (wid == 0) {
    unsigned key[2], at[2];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const uint2 t = lane < NT / 32 ? best[kind][lane] : make_uint2(0u, 0x7fffffffu);
      key[kind] = __reduce_max_sync(0xffffffffu, t.x);
      at[kind] = __reduce_min_sync(0xffffffffu, t.x == key[kind] ? t.y : 0x7fffffffu);
    }
    if (key[0] != 0u) {                            // which of the 16 bytes' tokens it was: a lane each
      const int e = (int)at[0] + lane;
      const bool in = lane < PER && ((pass8[e >> 3] >> (e & 7)) & 1u);
      const unsigned hit = __ballot_sync(0xffffffffu, in && ru_key(to_f(xs[in ? e : 0])) == key[0]);
      at[0] += __ffs(hit) - 1;
    }
    const bool stream = key[0] > key[1] || (key[0] == key[1] && at[0] < at[1]);
    const unsigned top = stream ? key[0] : key[1];
    const float v = top == 0u ? -INFINITY : __uint_as_float((top & 0x80000000u) ? top & 0x7fffffffu : ~top);
    const int i = top == 0u ? 0x7fffffff : e0 + (int)(stream ? at[0] : at[1]);
    if (lane == 0) {
      if constexpr (CL == 1) {
        A.choice[row] = i == 0x7fffffff ? 0 : i;
      } else {                                     // the slice's result to the shared memory of the cluster's first CTA
        uint32_t rv, ri;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rv) : "r"(smem_u32(&cv[rank])), "r"(0));
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ri) : "r"(smem_u32(&ci[rank])), "r"(0));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(rv), "f"(v) : "memory");
        asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(ri), "r"(i) : "memory");
      }
    }
  }
  if constexpr (CL > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && tid == 0) {
      float fv = -INFINITY;
      int fi = 0x7fffffff;
#pragma unroll
      for (int j = 0; j < CL; ++j) best_of(cv[j], ci[j], fv, fi);
      A.choice[row] = fi == 0x7fffffff ? 0 : fi;
    }
  }
}

// Adds tokens to the record: their bit, and with counts their number. Integer atomics: the order does not matter.
__global__ void __launch_bounds__(256) token_record_kernel(int* counts, unsigned* seen, const int* tok, const int* n_tok, int cap, int V, int words) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  const int n = n_tok ? min(cap, n_tok[b]) : cap;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int t = tok[(size_t)b * cap + i];
    if (t < 0 || t >= V) continue;
    if (seen) atomicOr(&seen[(size_t)b * words + (t >> 5)], 1u << (t & 31));
    if (counts) atomicAdd(&counts[(size_t)b * V + t], 1);
  }
}

}  // namespace moa
