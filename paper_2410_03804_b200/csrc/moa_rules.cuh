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
// record knows a few thousand of 128256 tokens. A CTA first makes a bitmap of its slice in shared memory, of the tokens that
// any rule but the mask touches (the record's bits, the path, the biases), with path and biases in a small hash table.
// Pass 1 streams the logits and looks at bits only. Pass 2 takes the marked tokens, whose counts are scattered loads: side
// by side over the CTA's threads. (Handled inside pass 1 they were one dependent load after the other for every warp that
// met a marked token: 281 us for 976 rows of 128256 bf16 with 300 biases.)
#pragma once
#include "moa_verify.cuh"

namespace moa {

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

template <typename T, int CL, int NT>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT) rules_kernel(const RulesArgs A) {
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
  const int n_words = (e1 - e0 + 31) >> 5;
  // shared memory: hash table (id, path count, bias entries, lowest of them, bias), then the slice's bitmap
  int* h_id = reinterpret_cast<int*>(ru_smem);
  int* h_cnt = h_id + A.table;
  int* h_n = h_cnt + A.table;
  int* h_first = h_n + A.table;
  float* h_val = reinterpret_cast<float*>(h_first + A.table);
  uint32_t* mark = reinterpret_cast<uint32_t*>(h_val + A.table);
  const unsigned hmask = A.table > 0 ? (unsigned)A.table - 1u : 0u;
  // every CTA of the cluster is running before another writes to its shared memory (waited for at the end)
  if constexpr (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  pdl_wait();

  const int* counts = A.counts ? A.counts + (size_t)b * A.V : nullptr;
  const unsigned* seen = A.seen ? A.seen + (size_t)b * A.words + (e0 >> 5) : nullptr;
  const unsigned* allow = A.allow ? A.allow + (size_t)row * A.words + (e0 >> 5) : nullptr;
  const bool dense = counts && !seen;        // counts without the record's bits: every count is read
  // ---- bitmap and hash table ----
  if (dense) {
    for (int i = tid; i < ((e1 - e0 + 31) & ~31); i += NT) {          // whole warps
      const unsigned m = __ballot_sync(0xffffffffu, e0 + i < e1 && counts[min(e0 + i, A.V - 1)] > 0);
      if ((i & 31) == 0) mark[i >> 5] = m;
    }
  } else {
    for (int i = tid; i < n_words; i += NT) mark[i] = seen ? __ldg(seen + i) : 0u;
  }
  if (A.table > 0) {
    for (int i = tid; i < A.table; i += NT) { h_id[i] = -1; h_cnt[i] = 0; h_n[i] = 0; h_first[i] = 0x7fffffff; }
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
    auto slot_of = [&](int id) {             // the table has at least twice the slots that can be asked for
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
      const int id = __ldg(bid + i);
      if (id < e0 || id >= e1) continue;
      const int s = slot_of(id);
      atomicAdd(&h_n[s], 1);
      atomicMin(&h_first[s], i);
      atomicOr(&mark[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    __syncthreads();
    const int np = s_np;
    for (int i = tid; i < np; i += NT) {
      const int id = s_path[i];
      if (id < e0 || id >= e1) continue;
      atomicAdd(&h_cnt[slot_of(id)], 1);
      atomicOr(&mark[(id - e0) >> 5], 1u << ((id - e0) & 31));
    }
    for (int s = tid; s < A.table; s += NT) {          // (the path only adds entries without a bias)
      if (h_n[s] == 0) continue;
      const int i0 = h_first[s], id = h_id[s];
      float v = __ldg(bval + i0);
      if (h_n[s] > 1)                        // the same id twice: summed in list order, whatever order the threads came in
        for (int i = i0 + 1; i < A.n_bias; ++i)
          if (__ldg(bid + i) == id) v = __fadd_rn(v, __ldg(bval + i));
      h_val[s] = v;
    }
  }
  __syncthreads();

  // ---- pass 1: the stream; marked tokens are written as they are and left out of the arg-max ----
  const T* xr = (const T*)A.x + (size_t)row * A.V;
  T* orow = A.out ? (T*)A.out + (size_t)row * A.V : nullptr;
  const uint8_t* mark8 = reinterpret_cast<const uint8_t*>(mark);
  const uint8_t* allow8 = reinterpret_cast<const uint8_t*>(allow);
  constexpr int PER = 16 / sizeof(T);
  constexpr unsigned ALL = (1u << PER) - 1u;
  float bv = -INFINITY;
  int bi = 0x7fffffff;
  const bool vec = ((reinterpret_cast<uintptr_t>(xr) | reinterpret_cast<uintptr_t>(orow)) & 15u) == 0;
  const int nvec = vec ? (e1 - e0) / PER : 0;
  constexpr int UN = 4;
  for (int c0 = tid; c0 < nvec; c0 += UN * NT) {
    uint4 raw[UN];
    unsigned ba[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int c = c0 + u * NT;
      const bool in = c < nvec;
      raw[u] = in ? __ldcs(reinterpret_cast<const uint4*>(xr + e0) + c) : make_uint4(0u, 0u, 0u, 0u);
      ba[u] = (in && allow8) ? (unsigned)__ldg(allow8 + (c * PER >> 3)) >> (PER == 4 ? (c * PER & 4) : 0) : ALL;
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int c = c0 + u * NT;
      if (c >= nvec) continue;
      const unsigned mk = ((unsigned)mark8[c * PER >> 3] >> (PER == 4 ? (c * PER & 4) : 0)) & ALL, al = ba[u] & ALL;
      float x[PER];
      if constexpr (sizeof(T) == 4) {
        x[0] = __uint_as_float(raw[u].x); x[1] = __uint_as_float(raw[u].y);
        x[2] = __uint_as_float(raw[u].z); x[3] = __uint_as_float(raw[u].w);
      } else {
        bf16x8_to_float(raw[u], x);
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
      if (mk != 0u) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if ((mk >> i) & 1u) x[i] = -INFINITY;
      }
      // a thread meets its elements in rising order, so "strictly greater" keeps the smallest id
      float vm = x[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) vm = fmaxf(vm, x[i]);
      if (vm > bv) {
        bv = vm;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
          if (x[i] == vm) bi = e0 + c * PER + i;
      }
    }
  }
  for (int i = nvec * PER + tid; i < e1 - e0; i += NT) {
    const bool al = !allow8 || ((__ldg(allow8 + (i >> 3)) >> (i & 7)) & 1u);
    const bool mk = (mark8[i >> 3] >> (i & 7)) & 1u;
    const float x = al ? to_f(xr[e0 + i]) : -INFINITY;
    if (orow) orow[e0 + i] = from_f<T>(x);
    if (!mk && x > bv) { bv = x; bi = e0 + i; }
  }
  __syncthreads();                           // pass 2 writes single elements over the vectors of pass 1

  // ---- pass 2: the marked tokens that are allowed ----
  const float rep = A.rep ? A.rep[b] : 1.f, freq = A.freq ? A.freq[b] : 0.f, pres = A.pres ? A.pres[b] : 0.f;
  for (int wi = tid; wi < n_words; wi += NT) {
    unsigned m = mark[wi];
    if (m == 0u) continue;
    if (allow) m &= __ldg(allow + wi);
    const unsigned in_record = seen ? __ldg(seen + wi) : 0u;
    while (m != 0u) {
      const int j = __ffs(m) - 1;
      m &= m - 1u;
      const int e = e0 + wi * 32 + j;
      if (e >= e1) break;                    // bits behind the vocabulary
      float x = to_f(xr[e]);
      bool known = (in_record >> j) & 1u;
      int c = 0;
      if (counts && (known || dense)) { c = __ldg(counts + e); known = known || c > 0; }
      bool biased = false;
      float bias = 0.f;
      if (A.table > 0) {
        for (unsigned s = ru_hash(e, hmask);; s = (s + 1u) & hmask) {
          const int id = h_id[s];
          if (id == -1) break;
          if (id == e) {
            c += h_cnt[s];
            known = known || h_cnt[s] > 0;
            biased = h_n[s] > 0;
            bias = h_val[s];
            break;
          }
        }
      }
      if (known && A.rep) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
      if (c > 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, (float)c)), pres);
      if (biased) x = __fadd_rn(x, bias);
      if (orow) orow[e] = from_f<T>(x);
      best_of(x, e, bv, bi);
    }
  }
  if (bv == -INFINITY) bi = 0x7fffffff;      // nothing above -inf: token 0, below

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
    bv = lane < NT / 32 ? sv[lane] : -INFINITY;
    bi = lane < NT / 32 ? si[lane] : 0x7fffffff;
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
