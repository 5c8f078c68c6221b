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
// record knows a few thousand of 128256 tokens. So the stream reads one bit per token of the record and of the mask; only a
// set bit leads to the token's count. Path tokens and biases of a CTA's slice go into a small hash table in shared memory
// behind a bitmap of the slice.
#pragma once
#include "moa_verify.cuh"

namespace moa {

constexpr int RU_THREADS = 256;
constexpr int RU_MAX_PATH = 256;             // tree slots per sequence
constexpr int RU_MAX_BIAS = 1024;

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

struct RuRow {                               // what one row's elements need
  const int* counts;
  const uint8_t *seen, *allow;
  float rep, freq, pres;
  bool has_rep;
};

template <typename T, int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(RU_THREADS) rules_kernel(const RulesArgs A) {
  pdl_trigger();
  extern __shared__ __align__(16) uint32_t ru_smem[];
  __shared__ float sv[32];
  __shared__ int si[32];
  __shared__ float cv[CL];
  __shared__ int ci[CL];
  __shared__ int s_path[RU_MAX_PATH], s_tok[RU_MAX_PATH], s_par[RU_MAX_PATH];
  __shared__ int s_np;
  const int rank = blockIdx.x, row = blockIdx.y, b = row / A.n, ti = row - b * A.n;
  const int tid = threadIdx.x;
  const int per_cta = ((A.V + CL - 1) / CL + 31) & ~31;
  const int e0 = min(A.V, rank * per_cta), e1 = min(A.V, e0 + per_cta);
  // shared memory: hash table (id, first entry / path count, value), then the slice's bitmap
  int* h_id = reinterpret_cast<int*>(ru_smem);
  int* h_cnt = h_id + A.table;               // occurrences on the path
  int* h_n = h_cnt + A.table;                // entries of the bias list
  int* h_first = h_n + A.table;              // the lowest of them
  float* h_val = reinterpret_cast<float*>(h_first + A.table);
  uint32_t* touch = reinterpret_cast<uint32_t*>(h_val + A.table);
  const unsigned hmask = A.table > 0 ? (unsigned)A.table - 1u : 0u;
  // every CTA of the cluster is running before another writes to its shared memory (waited for at the end)
  if constexpr (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  pdl_wait();

  if (A.table > 0) {
    for (int i = tid; i < A.table; i += RU_THREADS) { h_id[i] = -1; h_cnt[i] = 0; h_n[i] = 0; h_first[i] = 0x7fffffff; h_val[i] = 0.f; }
    for (int i = tid; i < per_cta / 32; i += RU_THREADS) touch[i] = 0u;
    if (A.tok)
      for (int i = tid; i < A.n; i += RU_THREADS) { s_tok[i] = A.tok[(size_t)b * A.n + i]; s_par[i] = A.parent[(size_t)b * A.n + i]; }
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
    __syncthreads();
    auto slot_of = [&](int id) {             // the table has at least twice the slots that can be asked for
      unsigned s = ru_hash(id, hmask);
      while (true) {
        const int old = atomicCAS(&h_id[s], -1, id);
        if (old == -1 || old == id) return (int)s;
        s = (s + 1u) & hmask;
      }
    };
    const int np = s_np;
    for (int i = tid; i < np; i += RU_THREADS) {
      const int id = s_path[i];
      if (id < e0 || id >= e1) continue;
      atomicAdd(&h_cnt[slot_of(id)], 1);
      atomicOr(&touch[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    const int* bid = A.bias_id + (size_t)b * A.n_bias;
    const float* bval = A.bias_val + (size_t)b * A.n_bias;
    for (int i = tid; i < A.n_bias; i += RU_THREADS) {
      const int id = bid[i];
      if (id < e0 || id >= e1) continue;
      const int s = slot_of(id);
      atomicAdd(&h_n[s], 1);
      atomicMin(&h_first[s], i);
      atomicOr(&touch[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    __syncthreads();
    for (int s = tid; s < A.table; s += RU_THREADS) {
      if (h_n[s] == 0) continue;
      const int i0 = h_first[s];
      float v = bval[i0];
      if (h_n[s] > 1)                        // the same id twice: summed in list order, whatever order the threads came in
        for (int i = i0 + 1; i < A.n_bias; ++i)
          if (bid[i] == h_id[s]) v = __fadd_rn(v, bval[i]);
      h_val[s] = v;
    }
    __syncthreads();
  }

  RuRow w;
  w.counts = A.counts ? A.counts + (size_t)b * A.V : nullptr;
  w.seen = A.seen ? reinterpret_cast<const uint8_t*>(A.seen + (size_t)b * A.words) : nullptr;
  w.allow = A.allow ? reinterpret_cast<const uint8_t*>(A.allow + (size_t)row * A.words) : nullptr;
  w.has_rep = A.rep != nullptr;
  w.rep = A.rep ? A.rep[b] : 1.f;
  w.freq = A.freq ? A.freq[b] : 0.f;
  w.pres = A.pres ? A.pres[b] : 0.f;
  const bool dense = w.counts && !w.seen;    // counts without the record's bits: every count is read
  const uint8_t* touch8 = reinterpret_cast<const uint8_t*>(touch);

  // one logit; known / touched / allowed: its bits
  auto rule = [&](float x, int e, bool known, bool touched, bool allowed) -> float {
    if (!allowed) return -INFINITY;
    int c = 0;
    if (w.counts && (known || dense)) { c = w.counts[e]; known = known || (dense && c > 0); }
    bool biased = false;
    float bias = 0.f;
    if (touched) {
      unsigned s = ru_hash(e, hmask);
      while (h_id[s] != e) s = (s + 1u) & hmask;          // the bit says that it is there
      const int on = h_cnt[s];
      c += on;
      known = known || on > 0;
      biased = h_n[s] > 0;
      bias = h_val[s];
    }
    if (known && w.has_rep) x = x > 0.f ? __fdiv_rn(x, w.rep) : __fmul_rn(x, w.rep);
    if (c > 0) {
      x = __fsub_rn(x, __fmul_rn(w.freq, (float)c));
      x = __fsub_rn(x, w.pres);
    }
    return biased ? __fadd_rn(x, bias) : x;
  };

  const T* xr = (const T*)A.x + (size_t)row * A.V;
  T* orow = A.out ? (T*)A.out + (size_t)row * A.V : nullptr;
  constexpr int PER = 16 / sizeof(T);
  float bv = -INFINITY;
  int bi = 0x7fffffff;
  const bool vec = ((reinterpret_cast<uintptr_t>(xr) | reinterpret_cast<uintptr_t>(orow)) & 15u) == 0;
  const int nvec = vec ? (e1 - e0) / PER : 0;
  constexpr int UN = 4;
  for (int c0 = tid; c0 < nvec; c0 += UN * RU_THREADS) {
    uint4 raw[UN];
    unsigned bs[UN], ba[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int c = c0 + u * RU_THREADS;
      const bool in = c < nvec;
      raw[u] = in ? __ldcs(reinterpret_cast<const uint4*>(xr + e0) + c) : make_uint4(0u, 0u, 0u, 0u);
      const int e = e0 + c * PER;
      const int sh = PER == 4 ? (e & 4) : 0;
      bs[u] = (in && w.seen) ? (unsigned)__ldg(w.seen + (e >> 3)) >> sh : 0u;
      ba[u] = (in && w.allow) ? (unsigned)__ldg(w.allow + (e >> 3)) >> sh : 0xffu;
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int c = c0 + u * RU_THREADS;
      if (c >= nvec) continue;
      const int e = e0 + c * PER;
      constexpr unsigned ALL = (1u << PER) - 1u;
      const unsigned bt = A.table > 0 ? ((unsigned)touch8[(e - e0) >> 3] >> (PER == 4 ? (e & 4) : 0)) & ALL : 0u;
      const unsigned kn = bs[u] & ALL, al = ba[u] & ALL;
      float x[PER];
      if constexpr (sizeof(T) == 4) {
        x[0] = __uint_as_float(raw[u].x); x[1] = __uint_as_float(raw[u].y);
        x[2] = __uint_as_float(raw[u].z); x[3] = __uint_as_float(raw[u].w);
      } else {
        bf16x8_to_float(raw[u], x);
      }
      if ((kn | bt) != 0u || dense) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if ((((kn | bt) >> i) & 1u) || dense) x[i] = rule(x[i], e + i, (kn >> i) & 1u, (bt >> i) & 1u, true);
      }
      if (al != ALL) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (!((al >> i) & 1u)) x[i] = -INFINITY;
      }
      if (orow) {
        uint4 y;
        if constexpr (sizeof(T) == 4) y = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        else y = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        __stcs(reinterpret_cast<uint4*>(orow + e0) + c, y);
      }
      // a thread meets its elements in rising order, so "strictly greater" keeps the smallest id
      float vm = x[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) vm = fmaxf(vm, x[i]);
      if (vm > bv) {
        bv = vm;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
          if (x[i] == vm) bi = e + i;
      }
    }
  }
  for (int e = e0 + nvec * PER + tid; e < e1; e += RU_THREADS) {
    const bool kn = w.seen && ((w.seen[e >> 3] >> (e & 7)) & 1u);
    const bool al = !w.allow || ((w.allow[e >> 3] >> (e & 7)) & 1u);
    const bool bt = A.table > 0 && ((touch8[(e - e0) >> 3] >> (e & 7)) & 1u);
    const float x = rule(to_f(xr[e]), e, kn, bt, al);
    if (orow) orow[e] = from_f<T>(x);
    if (x > bv) { bv = x; bi = e; }
  }
  if constexpr (CL > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (!A.choice) return;                     // the same for the whole grid
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
    const int oi = __shfl_xor_sync(0xffffffffu, bi, o);
    best_of(ov, oi, bv, bi);
  }
  const int lane = tid & 31, wid = tid >> 5;
  if (lane == 0) { sv[wid] = bv; si[wid] = bi; }
  __syncthreads();
  if (wid == 0) {
    bv = lane < RU_THREADS / 32 ? sv[lane] : -INFINITY;
    bi = lane < RU_THREADS / 32 ? si[lane] : 0x7fffffff;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
      const int oi = __shfl_xor_sync(0xffffffffu, bi, o);
      best_of(ov, oi, bv, bi);
    }
  }
  if constexpr (CL == 1) {
    if (tid == 0) A.choice[row] = bi == 0x7fffffff ? 0 : bi;
  } else {
    if (tid == 0) {                          // the slice's result to the shared memory of the cluster's first CTA
      uint32_t rv, ri;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rv) : "r"(smem_u32(&cv[rank])), "r"(0));
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ri) : "r"(smem_u32(&ci[rank])), "r"(0));
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(rv), "f"(bv) : "memory");
      asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(ri), "r"(bi) : "memory");
    }
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
