// Rows of logits: log probabilities of given tokens with entropy and top alternatives, distillation from a teacher's top
// logits, and the gradients of both.  For a row x of V logits at temperature tau
//     m = max_j x_j,  d_j = (x_j - m) / tau,  s = sum_j exp(d_j),  L = ln s,  p_j = exp(d_j - L)
//     logprob(id) = d_id - L,     H = L - sum_j exp(d_j) d_j / s
//     d logprob / dx_j = (1[j = id] - p_j) / tau,     dH / dx_j = -p_j (ln p_j + H) / tau
//     loss = sum_k q_k (ln q_k - ln p_{id_k}),  q = softmax(t / tau),     d loss / dx_j = (p_j - sum_{k: id_k = j} q_k) / tau
// Everything here moves a row through the chip once and does a handful of operations per logit, so DRAM bounds it.  A row (or, in a
// thread-block cluster, a CTA's part of it) is copied to shared memory asynchronously and stays there: the maximum, the sums with
// the maximum known, the alternatives and the gradient are passes over shared memory, and no pass rescales another's sums.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <cstdint>

#include "internal.h"
#include "sm100.cuh"   // the device status codes, cluster barriers

namespace fv {
namespace {

constexpr int kMaxAlt = 64;        // alternatives of a row
constexpr int kMaxTeacher = 128;   // entries of a teacher's row
constexpr int kMaxCluster = 8;     // CTAs that share a row
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---- small pieces -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) {   // 2^x within 2^-22 of its value, 0 at -inf, NaN at NaN
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float warp_max(float v) {   // NaN counts as absent
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_nctas() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t peer_smem(const void* p, uint32_t cta) {   // the same shared-memory address in another CTA of the cluster
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(cta));
  return r;
}
__device__ __forceinline__ void peer_store(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ void peer_store(uint32_t addr, uint64_t v) { asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory"); }
__device__ __forceinline__ void put_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}

// fp32 and bf16 logits: E elements in a 16-byte vector.
template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, uint64_t (&f)[2]) {
    f[0] = pack2(__uint_as_float(u.x), __uint_as_float(u.y));
    f[1] = pack2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&f)[2]) {
    float a, b, c, d;
    unpack2(f[0], a, b); unpack2(f[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
  static __device__ __forceinline__ float load(const float* p) { return dep_load(p); }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ float round(float v) { return v; }
  // running maximum of a thread
  struct Max {
    float m = -INFINITY;
    __device__ __forceinline__ void add(const uint4& u) {
      m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))));
    }
    __device__ __forceinline__ float value() const { return m; }
  };
  // whether a vector has an element of at least the threshold
  struct AtLeast {
    float t;
    __device__ __forceinline__ explicit AtLeast(float thr) : t(thr) {}
    __device__ __forceinline__ bool any(const uint4& u) const {
      return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))) >= t;
    }
  };
  static constexpr float kLowest = -FLT_MAX;
};
template <> struct Elem<__nv_bfloat16> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, uint64_t (&f)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      unpack2(f[i], lo, hi);
      w[i] = pack_bf16x2(lo, hi);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) {
    unsigned short v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return __uint_as_float((uint32_t)v << 16);
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
  static __device__ __forceinline__ __nv_bfloat162 b2(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  static __device__ __forceinline__ __nv_bfloat162 max4(const uint4& u) { return __hmax2(__hmax2(b2(u.x), b2(u.y)), __hmax2(b2(u.z), b2(u.w))); }
  struct Max {
    __nv_bfloat162 m = b2(0xFF80FF80u);   // -inf
    __device__ __forceinline__ void add(const uint4& u) { m = __hmax2(m, max4(u)); }
    __device__ __forceinline__ float value() const { return fmaxf(__low2float(m), __high2float(m)); }
  };
  struct AtLeast {
    __nv_bfloat162 t;
    __device__ __forceinline__ explicit AtLeast(float thr) : t(__float2bfloat162_rn(thr)) {}   // exact: thr is one of the row's values, or kLowest
    __device__ __forceinline__ bool any(const uint4& u) const { return !__hblt2(max4(u), t); }
  };
  static constexpr float kLowest = -3.3895313892515355e38f;
};

// An order of 32-bit integers that is the order of the values (-0 like +0; no NaN), above it the row's lowest index first: the key of an
// alternative.  0 is below every key of a finite value.
__device__ __forceinline__ uint64_t alt_key(float x, int idx) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (uint64_t)o << 32 | (0xFFFFFFFFu - (uint32_t)idx);
}
__device__ __forceinline__ float alt_value(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ int alt_index(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// ---- the part of a row that a group of G threads holds in shared memory ---------------------------------------------------
// Vectors of 16 bytes counted from the row's start rounded down to 16 bytes, so a row may start anywhere; elements of the first and last
// vector that are not the row's are -inf, which no pass notices.  The cluster's CTAs split the vectors evenly.  Thread t holds the
// vectors t, t + G, ... of its part; it alone copies, builds and reads them, so a row needs no barrier before it is used.
template <typename T, int G> struct Slice {
  static constexpr int E = Elem<T>::E;
  const T* row;      // first logit of the row
  int off, V;        // elements between the 16-byte boundary and the row; logits of the row
  int v0, n, t;      // first vector of this part, their number; thread of the group
  uint4* s;          // [n]
  __device__ __forceinline__ Slice(const T* row_, int V_, int rank, int parts, int t_, uint4* s_) : row(row_), V(V_), t(t_), s(s_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    const int nv = (off + V + E - 1) / E, base = nv / parts, rem = nv - base * parts;
    n = base + (rank < rem);
    v0 = rank * base + min(rank, rem);
  }
  __device__ __forceinline__ int first_index(int v) const { return (v0 + v) * E - off; }   // index in the row of the vector's first element
  __device__ __forceinline__ bool whole(int v) const { const int i = first_index(v); return i >= 0 && i + E <= V; }
  __device__ __forceinline__ void build(int v) {
    T* d = reinterpret_cast<T*>(s + v);
    const int i0 = first_index(v);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool in = i0 + e >= 0 && i0 + e < V;
      Elem<T>::store(d + e, in ? Elem<T>::load(row + i0 + e) : -INFINITY);
    }
  }
  __device__ __forceinline__ void fetch() {
    const char* g = reinterpret_cast<const char*>(row - off) + (size_t)v0 * 16;
    const uint32_t d = smem_u32(s);
    for (int v = t; v < n; v += G)
      if (whole(v)) cp_async16(d + v * 16, g + (size_t)v * 16);
    // the partial vectors: the row's first and last, where this part has them
    if (t == 0 && n > 0 && !whole(0)) build(0);
    if (n > 1 && (n - 1) % G == t && !whole(n - 1)) build(n - 1);
  }
};

template <int G> __device__ __forceinline__ void group_sync() {
  if constexpr (G == 32) __syncwarp();
  else __syncthreads();
}

// Sums with the maximum known: s = sum e, t = sum e d, e = 2^d, d = (x - m) log2(e) / tau.  The difference is taken before the product: x c - m c in
// one fused operation would be half an instruction per logit less, but rounds m c, which a row far from 0 (or masked with -1e9) makes larger than d.
struct Sums { float s, t; };
template <typename T, bool ENT> struct Summing {
  uint64_t c2, m2, s[2], t[2];
  __device__ __forceinline__ Summing(float c, float m) : c2(pack2(c, c)), m2(pack2(-m, -m)) { s[0] = s[1] = t[0] = t[1] = 0; }
  __device__ __forceinline__ void add(const uint4& u) {
    constexpr int P = Elem<T>::E / 2;
    uint64_t f[P];
    Elem<T>::unpack(u, f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t d = mul2(add2(f[i], m2), c2);
      float a, b;
      unpack2(d, a, b);
      const uint64_t e = pack2(exp2_fast(a), exp2_fast(b));
      s[i & 1] = add2(s[i & 1], e);
      if (ENT) t[i & 1] = fma2(e, pack2(fmaxf(a, -1e30f), fmaxf(b, -1e30f)), t[i & 1]);   // a logit of -inf adds 0, not 0 * -inf
    }
  }
  __device__ __forceinline__ Sums total() const {
    float a, b;
    unpack2(add2(s[0], s[1]), a, b);
    Sums r{a + b, 0.f};
    if (ENT) { unpack2(add2(t[0], t[1]), a, b); r.t = a + b; }
    return r;
  }
};

// What the parts of a row know of it, and what the whole row comes to.
struct Part { float m, s, t; };
struct Stat { float m, L, H, s; };
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }
template <bool ENT> __device__ __forceinline__ Stat stat_finish(const Part* parts, int n, float c) {
  Stat r;
  float s = parts[0].s, t = parts[0].t;
  r.m = parts[0].m;
  if (n > 1) {                          // a part's exponents were taken against its own maximum
    for (int i = 1; i < n; ++i) r.m = fmaxf(r.m, parts[i].m);
    const float m0 = safe_max(r.m);
    s = t = 0.f;
    for (int i = 0; i < n; ++i) {
      const float up = (safe_max(parts[i].m) - m0) * c, f = exp2_fast(up);
      if (parts[i].s == 0.f) continue;  // nothing but -inf (its up means nothing)
      s = fmaf(parts[i].s, f, s);
      if (ENT && f != 0.f) t = fmaf(fmaf(parts[i].s, up, parts[i].t), f, t);
    }
  }
  r.s = s;
  r.L = logf(s);
  r.H = ENT ? (s == 0.f ? 0.f : r.L - kLn2 * (t / s)) : 0.f;
  return r;
}

// ---- scratch of a group beside its slice ---------------------------------------------------------------------------------
constexpr int kThreadGroups = 128;                       // groups of threads whose maxima bound the alternatives from below (G > 32)
template <int G, bool ALT> struct alignas(16) Scratch {
  static constexpr int kCand = !ALT ? 0 : G == 32 ? 512 : 1024;
  float gm[ALT && G > 32 ? kThreadGroups : 4];
  float2 red[G / 32];
  float red_m[G / 32];
  float m, thr;
  int count;
  Part part[kMaxCluster];
  unsigned long long best[ALT ? G / 32 : 1];
  unsigned long long list[ALT ? kMaxAlt : 1];
  unsigned long long peers[ALT && G > 32 ? kMaxCluster * kMaxAlt : 1];   // the lists of the cluster's CTAs, in the first of them
  unsigned long long cand[kCand > 0 ? kCand : 1];
};

// The maximum of the group's part of the row, in every thread.
template <typename T, int G, bool ALT> __device__ __forceinline__ float part_max(const Slice<T, G>& sl, Scratch<G, ALT>& sc, float mine) {
  float m = warp_max(mine);
  if constexpr (G > 32) {
    const int warp = sl.t >> 5;
    if ((sl.t & 31) == 0) sc.red_m[warp] = m;
    __syncthreads();
    m = sc.red_m[0];
#pragma unroll
    for (int w = 1; w < G / 32; ++w) m = fmaxf(m, sc.red_m[w]);
  }
  return m;
}
// The same, and a value that at least n_alt of the part's elements reach: the n_alt-th largest among the maxima of 32 (a warp) or 128 groups of
// threads.  About n_alt (1 + n_alt / groups / 2) elements reach it where large values are spread over the row.  kLowest where fewer groups have a value.
template <typename T, int G> __device__ __forceinline__ float part_max_and_threshold(const Slice<T, G>& sl, Scratch<G, true>& sc, float mine, int n_alt, float& thr) {
  float m;
  if constexpr (G == 32) {
    int rank = 0;
    m = mine;
#pragma unroll
    for (int o = 1; o < 32; ++o) {
      const int src = (sl.t + o) & 31;
      const float v = __shfl_sync(0xFFFFFFFFu, mine, src);
      rank += v > mine || (v == mine && src < sl.t);
      m = fmaxf(m, v);
    }
    const uint32_t who = __ballot_sync(0xFFFFFFFFu, rank == n_alt - 1);
    thr = n_alt <= 32 ? __shfl_sync(0xFFFFFFFFu, mine, __ffs(who) - 1) : -INFINITY;
  } else {
    constexpr int SG = G / kThreadGroups;
    float g = mine;
#pragma unroll
    for (int o = SG / 2; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
    if (sl.t % SG == 0) sc.gm[sl.t / SG] = g;
    __syncthreads();
    if (sl.t < kThreadGroups) {
      const float my = sc.gm[sl.t];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < kThreadGroups; j += 4) {
        const float4 v = *reinterpret_cast<const float4*>(sc.gm + j);
        rank += (v.x > my || (v.x == my && j < sl.t)) + (v.y > my || (v.y == my && j + 1 < sl.t)) + (v.z > my || (v.z == my && j + 2 < sl.t)) +
                (v.w > my || (v.w == my && j + 3 < sl.t));
      }
      if (rank == 0) sc.m = my;
      if (rank == n_alt - 1) sc.thr = my;
    }
    __syncthreads();
    m = sc.m;
    thr = sc.thr;
  }
  thr = fmaxf(thr, Elem<T>::kLowest);     // -inf is never an alternative
  return m;
}

template <int G, bool ALT> __device__ __forceinline__ Sums part_sums(int t, Scratch<G, ALT>& sc, Sums mine, bool ent) {
  mine.s = warp_sum(mine.s);
  if (ent) mine.t = warp_sum(mine.t);
  if constexpr (G > 32) {
    if ((t & 31) == 0) sc.red[t >> 5] = make_float2(mine.s, mine.t);
    __syncthreads();
    mine = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < G / 32; ++w) { mine.s += sc.red[w].x; mine.t += sc.red[w].y; }
  } else {
    __syncwarp();
  }
  return mine;
}

template <typename T> __device__ __forceinline__ float slice_elem(const uint4* s, int v, int e) {
  if constexpr (sizeof(T) == 4) return reinterpret_cast<const float*>(s + v)[e];
  else return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(s + v)[e]);
}

// list[0 ... n_alt): the keys of the part's largest elements in descending order, 0 where there are fewer.  From the elements that reached the
// threshold, each ranked by counting; where there were too many to keep (rows of mostly equal values), by n_alt searches for the next largest key.
template <typename T, int G> __device__ __forceinline__ void part_list(const Slice<T, G>& sl, Scratch<G, true>& sc, int n_alt) {
  const int c = sc.count;
  if (c <= Scratch<G, true>::kCand) {
    for (int i = sl.t; i < c; i += G) {
      const unsigned long long key = sc.cand[i];
      int rank = 0;
      for (int j = 0; j < c; ++j) rank += sc.cand[j] > key;
      if (rank < n_alt) sc.list[rank] = key;
    }
  } else {
    unsigned long long prev = ~0ull;
    for (int a = 0; a < n_alt; ++a) {
      unsigned long long best = 0;
      for (int v = sl.t; v < sl.n; v += G) {
        const int i0 = sl.first_index(v);
#pragma unroll
        for (int e = 0; e < Elem<T>::E; ++e) {
          const float x = slice_elem<T>(sl.s, v, e);
          const unsigned long long key = x >= Elem<T>::kLowest ? alt_key(x, i0 + e) : 0;
          if (key < prev && key > best) best = key;
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, best, o);
        best = other > best ? other : best;
      }
      if constexpr (G > 32) {
        if ((sl.t & 31) == 0) sc.best[sl.t >> 5] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G / 32; ++w) best = sc.best[w] > best ? sc.best[w] : best;
        __syncthreads();
      }
      if (sl.t == 0) sc.list[a] = best;
      prev = best;
      if (best == 0) break;
    }
  }
  group_sync<G>();
}

// ---- log probabilities of given tokens, statistics, entropy, alternatives ------------------------------------------------
struct RowsArgs {
  const void* x; long long ld; int rows, V, per_max;   // per_max: vectors of the largest slice
  float inv_tau;
  const int32_t* ids; int n_alt;
  float* logprob; float2* stats; float* entropy; int32_t* alt_ids; float* alt_logprob;
  int32_t* status;
};

constexpr int kWarpRows = 4;       // rows of a CTA where a warp takes one
template <int G> constexpr int cta_threads() { return G == 32 ? 32 * kWarpRows : G; }
template <typename S> __host__ __device__ constexpr size_t group_bytes(int per_max) { return (size_t)per_max * 16 + sizeof(S); }

template <typename T, int G, bool ENT, bool ALT>
__global__ void __launch_bounds__(cta_threads<G>()) token_logprobs_kernel(const RowsArgs p) {
  using S = Scratch<G, ALT>;
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = G == 32 ? 1 : (int)cluster_nctas(), rank = G == 32 ? 0 : (int)cluster_ctarank();
  const int sub = G == 32 ? threadIdx.x >> 5 : 0, t = G == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int row = G == 32 ? blockIdx.x * kWarpRows + sub : blockIdx.x / parts;
  pdl_wait();
  if (G == 32 && row >= p.rows) return;
  if (G > 32 && parts > 1) cluster_arrive_relaxed();
  uint4* mine = reinterpret_cast<uint4*>(reinterpret_cast<char*>(smem) + sub * group_bytes<S>(p.per_max));
  S& sc = *reinterpret_cast<S*>(mine + p.per_max);
  const T* xrow = static_cast<const T*>(p.x) + row * p.ld;
  Slice<T, G> sl(xrow, p.V, rank, parts, t, mine);
  sl.fetch();
  float xid = 0.f;
  int id = -1;
  if (t == 0 && rank == 0 && p.ids) {
    id = dep_load(p.ids + row);
    if (id >= 0 && id < p.V) xid = Elem<T>::load(xrow + id);
  }
  if (ALT) {
    if (t < kMaxAlt) sc.list[t] = 0;
    if (G == 32) sc.list[t + 32] = 0;
    if (t == 0) sc.count = 0;
    if (G == 32) __syncwarp();
  }
  cp_async_wait_all();
  typename Elem<T>::Max mx;
  for (int v = t; v < sl.n; v += G) mx.add(mine[v]);
  float m, thr = 0.f;
  if constexpr (ALT) m = part_max_and_threshold<T, G>(sl, sc, mx.value(), p.n_alt, thr);
  else m = part_max<T, G, ALT>(sl, sc, mx.value());
  const float c = p.inv_tau * kLog2e;
  Summing<T, ENT> sum(c, safe_max(m));
  typename Elem<T>::AtLeast reach(thr);
#pragma unroll 2
  for (int v = t; v < sl.n; v += G) {
    const uint4 u = mine[v];
    sum.add(u);
    if (ALT && reach.any(u)) {
      const int i0 = sl.first_index(v);
      for (int e = 0; e < Elem<T>::E; ++e) {
        const float x = slice_elem<T>(mine, v, e);
        if (x >= thr) {
          const int slot = atomicAdd(&sc.count, 1);
          if (slot < S::kCand) sc.cand[slot] = alt_key(x, i0 + e);
        }
      }
    }
  }
  const Sums tot = part_sums<G, ALT>(t, sc, sum.total(), ENT);
  if constexpr (ALT) part_list<T, G>(sl, sc, p.n_alt);
  const Part part{m, tot.s, tot.t};
  Stat st;
  unsigned long long* alts = sc.list;
  if constexpr (G == 32) {
    st = stat_finish<ENT>(&part, 1, c);
  } else if (parts == 1) {
    st = stat_finish<ENT>(&part, 1, c);
  } else {
    __syncwarp();
    cluster_wait();                      // every CTA of the cluster has started
    if (t == 0) {
      const uint32_t to = peer_smem(&sc.part[rank], 0);
      peer_store(to, part.m); peer_store(to + 4, part.s); peer_store(to + 8, part.t);
    }
    if (ALT && t < p.n_alt) peer_store(peer_smem(&sc.peers[rank * kMaxAlt + t], 0), (uint64_t)sc.list[t]);
    __syncwarp();
    cluster_sync_all();
    if (rank != 0) return;
    st = stat_finish<ENT>(sc.part, parts, c);
    if constexpr (ALT) {                 // a key's place: its own, and how many of each other list are larger
      alts = sc.cand;
      if (t < p.n_alt) alts[t] = 0;
      __syncthreads();
      for (int i = t; i < parts * p.n_alt; i += G) {
        const int l = i / p.n_alt;
        int place = i - l * p.n_alt;
        const unsigned long long key = sc.peers[l * kMaxAlt + place];
        if (!key) continue;
        for (int o = 0; o < parts && place < p.n_alt; ++o) {
          if (o == l) continue;
          int lo = 0, hi = p.n_alt;
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (sc.peers[o * kMaxAlt + mid] > key) lo = mid + 1; else hi = mid;
          }
          place += lo;
        }
        if (place < p.n_alt) alts[place] = key;
      }
      __syncthreads();
    }
  }
  if (ALT)
    for (int i = t; i < p.n_alt; i += G) {
      const unsigned long long key = alts[i];
      const bool bad = st.L != st.L;
      const float lp = bad ? st.L : key ? (alt_value(key) - st.m) * p.inv_tau - st.L : -INFINITY;
      p.alt_ids[(size_t)row * p.n_alt + i] = bad || !key ? -1 : alt_index(key);
      p.alt_logprob[(size_t)row * p.n_alt + i] = lp;
    }
  if (t == 0) {
    if (p.stats) p.stats[row] = make_float2(st.m, st.L);
    if (ENT) p.entropy[row] = st.H;
    if (p.logprob) {
      float lp = 0.f;                    // -1: the row has no token
      if (id >= 0 && id < p.V) {
        lp = st.L == -INFINITY ? -INFINITY : (xid - st.m) * p.inv_tau - st.L;
      } else if (id != -1) {
        put_status(p.status, DEV_BAD_TOKEN_ID);
        lp = __int_as_float(0x7FC00000);
      }
      p.logprob[row] = lp;
    }
  }
}

// ---- distillation: loss, and with GRAD its gradient while the row is still in shared memory --------------------------------
struct DistillArgs {
  const void* x; long long ld; int rows, V, per_max;
  float inv_tau;
  const int32_t* t_ids; const float* t_logits; int K;
  const float* g;                  // [rows] or null: 1
  float* loss; float2* stats;
  void* dx; long long ld_dx;
  int32_t* status;
};

// The teacher's row: lane l of one warp holds the entries l, l + 32, ...; q over the entries that have a token (-1: none).
struct Teacher {
  static constexpr int P = kMaxTeacher / 32;
  int id[P];
  float q[P], lq[P];
  bool some, bad;
  __device__ __forceinline__ void load(const int32_t* ids, const float* logits, int K, int V, float inv_tau, int lane) {
    float x[P], m = -INFINITY;
    bool wrong = false, any = false;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int k = lane + 32 * i;
      id[i] = -1;
      x[i] = -INFINITY;
      if (k < K) {
        const int v = dep_load(ids + k);
        if (v >= 0 && v < V) {
          id[i] = v;
          x[i] = dep_load(logits + k);
        } else {
          wrong |= v != -1;
        }
      }
      any |= x[i] != -INFINITY;
      m = fmaxf(m, x[i]);
    }
    m = safe_max(warp_max(m));
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) { lq[i] = (x[i] - m) * inv_tau; q[i] = expf(lq[i]); s += q[i]; }
    s = warp_sum(s);
    some = __any_sync(0xFFFFFFFFu, any);
    bad = __any_sync(0xFFFFFFFFu, wrong);
    const float ls = logf(s);
#pragma unroll
    for (int i = 0; i < P; ++i) { q[i] = some ? q[i] / s : 0.f; lq[i] -= ls; }
  }
};
struct TeacherRow {                // of one row, for the gradient's corrections
  int id[kMaxTeacher];
  float q[kMaxTeacher], x[kMaxTeacher];
  int some;
};
// What entry k takes off its token's probability: all entries of that token together, at the first of them; -1 elsewhere.
__device__ __forceinline__ float teacher_share(const TeacherRow& tr, int k, int K) {
  const int id = tr.id[k];
  if (id < 0) return -1.f;
  float sum = 0.f;
  bool first = true;
  for (int j = 0; j < K; ++j) {
    const bool same = tr.id[j] == id;
    first &= !(same && j < k);
    sum += same ? tr.q[j] : 0.f;
  }
  return first ? sum : -1.f;
}

template <typename T> __device__ __forceinline__ bool same_alignment(const T* a, const T* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

template <typename T, int G, bool GRAD>
__global__ void __launch_bounds__(cta_threads<G>()) distill_kernel(const DistillArgs p) {
  struct alignas(16) S { Scratch<G, false> sc; TeacherRow tr; };
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = G == 32 ? 1 : (int)cluster_nctas(), rank = G == 32 ? 0 : (int)cluster_ctarank();
  const int sub = G == 32 ? threadIdx.x >> 5 : 0, t = G == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int row = G == 32 ? blockIdx.x * kWarpRows + sub : blockIdx.x / parts;
  pdl_wait();
  if (G == 32 && row >= p.rows) return;
  if (G > 32 && parts > 1) cluster_arrive_relaxed();
  uint4* mine = reinterpret_cast<uint4*>(reinterpret_cast<char*>(smem) + sub * group_bytes<S>(p.per_max));
  S& own = *reinterpret_cast<S*>(mine + p.per_max);
  Scratch<G, false>& sc = own.sc;
  TeacherRow& tr = own.tr;
  const T* xrow = static_cast<const T*>(p.x) + row * p.ld;
  Slice<T, G> sl(xrow, p.V, rank, parts, t, mine);
  sl.fetch();
  Teacher te;
  float xk[Teacher::P];
  if (t < 32 && (GRAD || rank == 0)) {
    te.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, p.V, p.inv_tau, t);
#pragma unroll
    for (int i = 0; i < Teacher::P; ++i) {
      xk[i] = te.id[i] >= 0 ? Elem<T>::load(xrow + te.id[i]) : 0.f;
      if (GRAD) { tr.id[t + 32 * i] = te.id[i]; tr.q[t + 32 * i] = te.q[i]; tr.x[t + 32 * i] = xk[i]; }
    }
    if (GRAD && t == 0) tr.some = te.some;
  }
  cp_async_wait_all();
  typename Elem<T>::Max mx;
  for (int v = t; v < sl.n; v += G) mx.add(mine[v]);
  const float m = part_max<T, G, false>(sl, sc, mx.value());
  const float c = p.inv_tau * kLog2e;
  Summing<T, false> sum(c, safe_max(m));
#pragma unroll 2
  for (int v = t; v < sl.n; v += G) sum.add(mine[v]);
  const Sums tot = part_sums<G, false>(t, sc, sum.total(), false);
  const Part part{m, tot.s, 0.f};
  Stat st;
  if (G == 32 || parts == 1) {
    st = stat_finish<false>(&part, 1, c);
  } else {
    __syncwarp();
    cluster_wait();
    if (t < (GRAD ? parts : 1)) {
      const uint32_t to = peer_smem(&sc.part[rank], t);
      peer_store(to, part.m); peer_store(to + 4, part.s); peer_store(to + 8, 0.f);
    }
    __syncwarp();
    cluster_sync_all();                  // in place: and every CTA has read the logits of the teacher's tokens
    if (!GRAD && rank != 0) return;
    st = stat_finish<false>(sc.part, parts, c);
  }
  if (rank == 0 && t < 32) {
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < Teacher::P; ++i) {
      const float lp = st.L == -INFINITY ? -INFINITY : (xk[i] - st.m) * p.inv_tau - st.L;
      if (te.id[i] >= 0 && te.q[i] != 0.f) loss = fmaf(te.q[i], te.lq[i] - lp, loss);   // (q NaN: the loss too)
    }
    loss = warp_sum(loss);
    if (t == 0) {
      if (te.bad) { put_status(p.status, DEV_BAD_TOKEN_ID); loss = __int_as_float(0x7FC00000); }
      p.loss[row] = loss;
      if (p.stats) p.stats[row] = make_float2(st.m, st.L);
    }
  }
  if constexpr (GRAD) {
    constexpr int E = Elem<T>::E, P = E / 2;
    T* drow = static_cast<T*>(p.dx) + row * p.ld_dx;
    const float w = (p.g ? dep_load(p.g + row) : 1.f) * p.inv_tau;
    const bool none = !tr.some || w == 0.f || st.L == -INFINITY;   // (tr: written before the barriers of the sums)
    const float f = none ? 0.f : w / st.s;
    const uint64_t c2 = pack2(c, c), m2 = pack2(-st.m, -st.m), f2 = pack2(f, f);
    const bool vec = same_alignment(xrow, drow);
    T* dvec = drow - sl.off + (size_t)sl.v0 * E;
#pragma unroll 2
    for (int v = t; v < sl.n; v += G) {
      uint64_t d[P];
      Elem<T>::unpack(mine[v], d);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float a, b;
        unpack2(mul2(add2(d[i], m2), c2), a, b);
        d[i] = none ? 0 : mul2(pack2(exp2_fast(a), exp2_fast(b)), f2);
      }
      if (vec && sl.whole(v)) {
        *reinterpret_cast<uint4*>(dvec + (size_t)v * E) = Elem<T>::pack(d);
      } else {
        const int i0 = sl.first_index(v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float a, b;
          unpack2(d[e >> 1], a, b);
          if (i0 + e >= 0 && i0 + e < p.V) Elem<T>::store(drow + i0 + e, e & 1 ? b : a);
        }
      }
    }
    group_sync<G>();
    if (!none)
      for (int k = t; k < p.K; k += G) {
        const int id = tr.id[k];
        const int at = id < 0 ? -1 : (id + sl.off) / E - sl.v0;
        if (at < 0 || at >= sl.n) continue;
        const float share = teacher_share(tr, k, p.K);
        if (share < 0.f) continue;
        Elem<T>::store(drow + id, fmaf(exp2_fast((tr.x[k] - st.m) * c), f, -w * share));
      }
  }
}

// ---- gradients for weights that come after the forward call ---------------------------------------------------------------
// One pass over the row with its statistics known.  A warp takes U vectors per lane of a row, all of them on their way before the first is
// used; no barrier and no shared memory, so 64 warps per SM keep DRAM busy.
struct GradArgs {
  const void* x; long long ld; int rows, V, segs;   // segs: warps per row
  float inv_tau;
  const float2* stats; const float* entropy; const int32_t* ids;
  const float* g_logprob; const float* g_entropy;
  const int32_t* t_ids; const float* t_logits; int K;
  void* dx; long long ld_dx;
  int32_t* status;
};
constexpr int kGradWarps = 8;

// The part of a row that a warp takes: where its vectors lie, what they hold, how they are written.
template <typename T, int U> struct Segment {
  static constexpr int E = Elem<T>::E;
  const T* row;
  T* drow;
  int off, V, v0, nv;   // v0: the lane's first vector; the others are 32 further each
  bool vec;
  __device__ __forceinline__ Segment(const T* row_, T* drow_, int V_, int seg, int lane) : row(row_), drow(drow_), V(V_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    nv = (off + V + E - 1) / E;
    v0 = seg * (32 * U) + lane;
    vec = same_alignment(row, static_cast<const T*>(drow));
  }
  __device__ __forceinline__ int first_index(int u) const { return (v0 + 32 * u) * E - off; }
  __device__ __forceinline__ bool whole(int u) const { const int i = first_index(u); return i >= 0 && i + E <= V; }
  __device__ __forceinline__ void load(uint4 (&x)[U]) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i0 = first_index(u);
      if (whole(u)) {
        x[u] = dep_load16(row + i0);
      } else if (v0 + 32 * u < nv) {
        uint64_t f[E / 2];
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const bool a = i0 + e >= 0 && i0 + e < V, b = i0 + e + 1 >= 0 && i0 + e + 1 < V;
          f[e / 2] = pack2(a ? Elem<T>::load(row + i0 + e) : 0.f, b ? Elem<T>::load(row + i0 + e + 1) : 0.f);
        }
        x[u] = Elem<T>::pack(f);
      }
    }
  }
  __device__ __forceinline__ void store(int u, const uint64_t (&d)[E / 2]) const {
    const int i0 = first_index(u);
    if (vec && whole(u)) {
      *reinterpret_cast<uint4*>(drow + i0) = Elem<T>::pack(d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float a, b;
        unpack2(d[e >> 1], a, b);
        if (i0 + e >= 0 && i0 + e < V) Elem<T>::store(drow + i0 + e, e & 1 ? b : a);
      }
    }
  }
  __device__ __forceinline__ void zero() const {
    uint64_t d[E / 2] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v0 + 32 * u < nv) store(u, d);
  }
};

// Two exponents of 2: log2 p of a pair of logits.
struct LogP {
  uint64_t neg_m, c, neg_L;
  __device__ __forceinline__ LogP(float m, float c_, float L2) : neg_m(pack2(-m, -m)), c(pack2(c_, c_)), neg_L(pack2(-L2, -L2)) {}
  __device__ __forceinline__ uint64_t operator()(uint64_t x) const { return fma2(add2(x, neg_m), c, neg_L); }
};

template <typename T, int U, bool ENT>
__global__ void __launch_bounds__(32 * kGradWarps) token_logprobs_grad_kernel(const GradArgs p) {
  constexpr int E = Elem<T>::E;
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * kGradWarps + (threadIdx.x >> 5);
  pdl_wait();
  const int row = (int)(unit / p.segs), seg = (int)(unit - (long long)row * p.segs);
  if (row >= p.rows) return;
  const Segment<T, U> sg(static_cast<const T*>(p.x) + row * p.ld, static_cast<T*>(p.dx) + row * p.ld_dx, p.V, seg, lane);
  uint4 x[U];
  sg.load(x);
  const float m = dep_load(&p.stats[row].x), L = dep_load(&p.stats[row].y);
  int id = p.ids ? dep_load(p.ids + row) : -1;
  if (id < 0 || id >= p.V) {
    if (id != -1 && seg == 0 && lane == 0) put_status(p.status, DEV_BAD_TOKEN_ID);
    id = -1;
  }
  const float gl = id >= 0 && p.g_logprob ? dep_load(p.g_logprob + row) * p.inv_tau : 0.f;
  const float ge = ENT ? dep_load(p.g_entropy + row) * p.inv_tau : 0.f;
  if ((gl == 0.f && ge == 0.f) || L == -INFINITY) {
    sg.zero();
    return;
  }
  const float A = ENT ? -fmaf(ge, dep_load(p.entropy + row), gl) : -gl, B = -ge * kLn2;   // dx = p (A + B log2 p), at the token + gl
  const LogP logp(m, p.inv_tau * kLog2e, L * kLog2e);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (sg.v0 + 32 * u >= sg.nv) break;
    uint64_t d[E / 2];
    Elem<T>::unpack(x[u], d);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      float a, b;
      unpack2(logp(d[i]), a, b);
      const uint64_t q = pack2(exp2_fast(a), exp2_fast(b));
      d[i] = mul2(q, ENT ? fma2(pack2(B, B), pack2(fmaxf(a, -1e4f), fmaxf(b, -1e4f)), pack2(A, A)) : pack2(A, A));   // (p = 0 below 2^-1e4)
    }
    const int at = id - sg.first_index(u);
    if (id >= 0 && at >= 0 && at < E) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float a, b;
        unpack2(d[e >> 1], a, b);
        if (e == at) d[e >> 1] = e & 1 ? pack2(a, b + gl) : pack2(a + gl, b);
      }
    }
    sg.store(u, d);
  }
}

template <typename T, int U>
__global__ void __launch_bounds__(32 * kGradWarps) distill_grad_kernel(const GradArgs p) {
  constexpr int E = Elem<T>::E;
  __shared__ TeacherRow teacher[kGradWarps];
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * kGradWarps + (threadIdx.x >> 5);
  TeacherRow& tr = teacher[threadIdx.x >> 5];
  pdl_wait();
  const int row = (int)(unit / p.segs), seg = (int)(unit - (long long)row * p.segs);
  if (row >= p.rows) return;
  const T* xrow = static_cast<const T*>(p.x) + row * p.ld;
  T* drow = static_cast<T*>(p.dx) + row * p.ld_dx;
  const Segment<T, U> sg(xrow, drow, p.V, seg, lane);
  uint4 x[U];
  sg.load(x);
  Teacher te;
  te.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, p.V, p.inv_tau, lane);
  if (te.bad && seg == 0 && lane == 0) put_status(p.status, DEV_BAD_TOKEN_ID);
  const float m = dep_load(&p.stats[row].x), L = dep_load(&p.stats[row].y);
  const float w = (p.g_logprob ? dep_load(p.g_logprob + row) : 1.f) * p.inv_tau;
  if (!te.some || w == 0.f || L == -INFINITY) {
    sg.zero();
    return;
  }
  const int lo = (seg * 32 * U) * E - sg.off, hi = min(p.V, lo + 32 * U * E);   // the logits of this warp
#pragma unroll
  for (int i = 0; i < Teacher::P; ++i) {
    const int id = te.id[i];
    tr.id[lane + 32 * i] = id;
    tr.q[lane + 32 * i] = te.q[i];
    if (id >= lo && id < hi) tr.x[lane + 32 * i] = Elem<T>::load(xrow + id);
  }
  __syncwarp();
  const float c = p.inv_tau * kLog2e, L2 = L * kLog2e;
  const LogP logp(m, c, L2);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (sg.v0 + 32 * u >= sg.nv) break;
    uint64_t d[E / 2];
    Elem<T>::unpack(x[u], d);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      float a, b;
      unpack2(logp(d[i]), a, b);
      d[i] = mul2(pack2(exp2_fast(a), exp2_fast(b)), pack2(w, w));
    }
    sg.store(u, d);
  }
  __syncwarp();
  for (int k = lane; k < p.K; k += 32) {
    const int id = tr.id[k];
    if (id < lo || id >= hi) continue;
    const float share = teacher_share(tr, k, p.K);
    if (share >= 0.f || share != share) Elem<T>::store(drow + id, w * (exp2_fast(fmaf(tr.x[k] - m, c, -L2)) - share));
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
int logits_vectors(int V, int E) { return (V + E - 1 + E - 1) / E; }   // most 16-byte vectors that a row touches

template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), unsigned grid, int threads, int cluster, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Who takes a row: a warp, or a cluster of CTAs of 256 threads.
struct Shape { int group, cluster, per_max; };
constexpr int kMaxRowBytes = 1536 << 10;
Shape row_shape(int rows, int V, int es, bool warp_may) {
  const int nv = logits_vectors(V, 16 / es);
  if (warp_may && nv <= 1024 && rows >= 148 * 8) return {32, 1, nv};
  int s = 1;
  while (s < kMaxCluster && (size_t)(nv + s - 1) / s * 16 > (48 << 10)) s *= 2;
  while (s < kMaxCluster && (long long)rows * s < 148 && nv / (2 * s) >= 512) s *= 2;
  return {256, s, (nv + s - 1) / s};
}

constexpr int kMaxSmem = 227 << 10;
template <typename K> cudaError_t allow_smem(K kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem); }
template <typename T> cudaError_t allow_all() {
  cudaError_t e = cudaSuccess;
  auto add = [&](auto kernel) { if (e == cudaSuccess) e = allow_smem(kernel); };
  add(token_logprobs_kernel<T, 32, false, false>); add(token_logprobs_kernel<T, 32, false, true>);
  add(token_logprobs_kernel<T, 32, true, false>); add(token_logprobs_kernel<T, 32, true, true>);
  add(token_logprobs_kernel<T, 256, false, false>); add(token_logprobs_kernel<T, 256, false, true>);
  add(token_logprobs_kernel<T, 256, true, false>); add(token_logprobs_kernel<T, 256, true, true>);
  add(distill_kernel<T, 32, false>); add(distill_kernel<T, 32, true>);
  add(distill_kernel<T, 256, false>); add(distill_kernel<T, 256, true>);
  return e;
}
// Function attributes belong to a device: set on the first call on each.
cudaError_t logits_init() {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1))) return e;
  e = allow_all<float>();
  if (e == cudaSuccess) e = allow_all<__nv_bfloat16>();
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return e;
}

template <typename T, int G, bool ENT, bool ALT> cudaError_t go_token(RowsArgs& a, const Shape& s, cudaStream_t st) {
  const size_t smem = group_bytes<Scratch<G, ALT>>(s.per_max) * (G == 32 ? kWarpRows : 1);
  const unsigned grid = G == 32 ? (a.rows + kWarpRows - 1) / kWarpRows : (unsigned)a.rows * s.cluster;
  return launch_clusters(token_logprobs_kernel<T, G, ENT, ALT>, grid, cta_threads<G>(), s.cluster, smem, st, a);
}
template <typename T> cudaError_t launch_token(RowsArgs& a, cudaStream_t st) {
  const Shape s = row_shape(a.rows, a.V, sizeof(T), a.n_alt <= 24);
  a.per_max = s.per_max;
  const bool ent = a.entropy != nullptr, alt = a.n_alt > 0;
  if (s.group == 32)
    return ent ? (alt ? go_token<T, 32, true, true>(a, s, st) : go_token<T, 32, true, false>(a, s, st))
               : (alt ? go_token<T, 32, false, true>(a, s, st) : go_token<T, 32, false, false>(a, s, st));
  return ent ? (alt ? go_token<T, 256, true, true>(a, s, st) : go_token<T, 256, true, false>(a, s, st))
             : (alt ? go_token<T, 256, false, true>(a, s, st) : go_token<T, 256, false, false>(a, s, st));
}
template <typename T, int G, bool GRAD> cudaError_t go_distill(DistillArgs& a, const Shape& s, cudaStream_t st) {
  struct alignas(16) S { Scratch<G, false> sc; TeacherRow tr; };   // as in the kernel
  const size_t smem = group_bytes<S>(s.per_max) * (G == 32 ? kWarpRows : 1);
  const unsigned grid = G == 32 ? (a.rows + kWarpRows - 1) / kWarpRows : (unsigned)a.rows * s.cluster;
  return launch_clusters(distill_kernel<T, G, GRAD>, grid, cta_threads<G>(), s.cluster, smem, st, a);
}
template <typename T> cudaError_t launch_distill(DistillArgs& a, cudaStream_t st) {
  const Shape s = row_shape(a.rows, a.V, sizeof(T), true);
  a.per_max = s.per_max;
  if (s.group == 32) return a.dx ? go_distill<T, 32, true>(a, s, st) : go_distill<T, 32, false>(a, s, st);
  return a.dx ? go_distill<T, 256, true>(a, s, st) : go_distill<T, 256, false>(a, s, st);
}
template <typename T, int U, typename K> cudaError_t launch_grad(K kernel, GradArgs& a, cudaStream_t st) {
  a.segs = (logits_vectors(a.V, Elem<T>::E) + 32 * U - 1) / (32 * U);
  const long long ctas = ((long long)a.rows * a.segs + kGradWarps - 1) / kGradWarps;
  if (ctas > INT_MAX) return cudaErrorInvalidValue;
  return launch_pdl(kernel, dim3((unsigned)ctas), dim3(32 * kGradWarps), 0, st, a);
}

bool al(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// Logits of either type: a size, a stride and an address that the kernels take.
fv_status check_rows(const void* x, int32_t dtype, int64_t ld, int32_t rows, int32_t V, float tau) {
  if (!x || rows <= 0 || V <= 0 || ld < V || (dtype != 0 && dtype != 1) || !(tau >= 1e-6f && tau <= 1e6f)) return FV_ERR_INVALID_ARG;
  const size_t es = dtype ? 2 : 4;
  if (!al(x, es)) return FV_ERR_INVALID_ARG;
  if ((size_t)V * es > (size_t)kMaxRowBytes || (long long)rows * kMaxCluster > INT_MAX) return FV_ERR_UNSUPPORTED;
  return FV_OK;
}
fv_status cu(cudaError_t e) { return e == cudaSuccess ? FV_OK : FV_ERR_CUDA; }

}  // namespace
}  // namespace fv

using namespace fv;

extern "C" {

fv_status fv_token_logprobs(const void* logits_dev, int32_t dtype, int64_t ld, int32_t rows, int32_t V, float tau, const int32_t* ids_dev,
                            int32_t n_alt, float* logprob_out_dev, float* stats_out_dev, float* entropy_out_dev, int32_t* alt_ids_out_dev,
                            float* alt_logprob_out_dev, int32_t* status_dev, void* stream) {
  const fv_status s = check_rows(logits_dev, dtype, ld, rows, V, tau);
  if (s != FV_OK) return s;
  if (n_alt < 0 || n_alt > kMaxAlt || (n_alt > 0) != (alt_ids_out_dev != nullptr) || (n_alt > 0) != (alt_logprob_out_dev != nullptr)) return FV_ERR_INVALID_ARG;
  if ((ids_dev != nullptr) != (logprob_out_dev != nullptr) || !al(stats_out_dev, 8)) return FV_ERR_INVALID_ARG;
  if (!logprob_out_dev && !stats_out_dev && !entropy_out_dev && n_alt == 0) return FV_ERR_INVALID_ARG;
  if (logits_init() != cudaSuccess) return FV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const double bytes = (double)rows * ((dtype ? 2.0 : 4.0) * V + 20.0 + 8.0 * n_alt);
  LaunchScope scope(KC_SELECT, 1, bytes, bytes, st);
  RowsArgs a{logits_dev, ld, rows, V, 0, 1.f / tau, ids_dev, n_alt, logprob_out_dev, reinterpret_cast<float2*>(stats_out_dev), entropy_out_dev,
             alt_ids_out_dev, alt_logprob_out_dev, status_dev};
  return cu(dtype ? launch_token<__nv_bfloat16>(a, st) : launch_token<float>(a, st));
}

fv_status fv_token_logprobs_grad(const void* logits_dev, int32_t dtype, int64_t ld, int32_t rows, int32_t V, float tau, const int32_t* ids_dev,
                                 const float* stats_dev, const float* entropy_dev, const float* g_logprob_dev, const float* g_entropy_dev,
                                 void* dlogits_out_dev, int64_t ld_out, int32_t* status_dev, void* stream) {
  const fv_status s = check_rows(logits_dev, dtype, ld, rows, V, tau);
  if (s != FV_OK) return s;
  if (!stats_dev || !al(stats_dev, 8) || !dlogits_out_dev || !al(dlogits_out_dev, dtype ? 2 : 4) || ld_out < V) return FV_ERR_INVALID_ARG;
  if ((ids_dev != nullptr) != (g_logprob_dev != nullptr) || (g_entropy_dev && !entropy_dev) || (!g_logprob_dev && !g_entropy_dev)) return FV_ERR_INVALID_ARG;
  if (dlogits_out_dev == logits_dev && ld_out != ld) return FV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const double bytes = (double)rows * ((dtype ? 4.0 : 8.0) * V + 24.0);
  LaunchScope scope(KC_SELECT, 1, bytes, bytes, st);
  GradArgs a{logits_dev, ld, rows, V, 0, 1.f / tau, reinterpret_cast<const float2*>(stats_dev), entropy_dev, ids_dev, g_logprob_dev, g_entropy_dev,
             nullptr, nullptr, 0, dlogits_out_dev, ld_out, status_dev};
  using B = __nv_bfloat16;
  if (dtype) return cu(g_entropy_dev ? launch_grad<B, 4>(token_logprobs_grad_kernel<B, 4, true>, a, st) : launch_grad<B, 4>(token_logprobs_grad_kernel<B, 4, false>, a, st));
  return cu(g_entropy_dev ? launch_grad<float, 4>(token_logprobs_grad_kernel<float, 4, true>, a, st) : launch_grad<float, 4>(token_logprobs_grad_kernel<float, 4, false>, a, st));
}

fv_status fv_distill_topk(const void* logits_dev, int32_t dtype, int64_t ld, int32_t rows, int32_t V, float tau, const int32_t* teacher_ids_dev,
                          const float* teacher_logits_dev, int32_t K, const float* g_loss_dev, float* loss_out_dev, float* stats_out_dev,
                          void* dlogits_out_dev, int64_t ld_out, int32_t* status_dev, void* stream) {
  const fv_status s = check_rows(logits_dev, dtype, ld, rows, V, tau);
  if (s != FV_OK) return s;
  if (!teacher_ids_dev || !teacher_logits_dev || K <= 0 || K > kMaxTeacher || !loss_out_dev || !al(stats_out_dev, 8)) return FV_ERR_INVALID_ARG;
  if (dlogits_out_dev ? !al(dlogits_out_dev, dtype ? 2 : 4) || ld_out < V || (dlogits_out_dev == logits_dev && ld_out != ld) : g_loss_dev != nullptr) return FV_ERR_INVALID_ARG;
  if (logits_init() != cudaSuccess) return FV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const double bytes = (double)rows * ((dtype ? 2.0 : 4.0) * V * (dlogits_out_dev ? 2.0 : 1.0) + 8.0 * K + 16.0);
  LaunchScope scope(KC_SELECT, 1, bytes, bytes, st);
  DistillArgs a{logits_dev, ld, rows, V, 0, 1.f / tau, teacher_ids_dev, teacher_logits_dev, K, g_loss_dev, loss_out_dev, reinterpret_cast<float2*>(stats_out_dev),
                dlogits_out_dev, ld_out, status_dev};
  return cu(dtype ? launch_distill<__nv_bfloat16>(a, st) : launch_distill<float>(a, st));
}

fv_status fv_distill_topk_grad(const void* logits_dev, int32_t dtype, int64_t ld, int32_t rows, int32_t V, float tau, const int32_t* teacher_ids_dev,
                               const float* teacher_logits_dev, int32_t K, const float* stats_dev, const float* g_loss_dev, void* dlogits_out_dev,
                               int64_t ld_out, int32_t* status_dev, void* stream) {
  const fv_status s = check_rows(logits_dev, dtype, ld, rows, V, tau);
  if (s != FV_OK) return s;
  if (!teacher_ids_dev || !teacher_logits_dev || K <= 0 || K > kMaxTeacher || !stats_dev || !al(stats_dev, 8)) return FV_ERR_INVALID_ARG;
  if (!dlogits_out_dev || !al(dlogits_out_dev, dtype ? 2 : 4) || ld_out < V || (dlogits_out_dev == logits_dev && ld_out != ld)) return FV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const double bytes = (double)rows * ((dtype ? 4.0 : 8.0) * V + 8.0 * K + 12.0);
  LaunchScope scope(KC_SELECT, 1, bytes, bytes, st);
  GradArgs a{logits_dev, ld, rows, V, 0, 1.f / tau, reinterpret_cast<const float2*>(stats_dev), nullptr, nullptr, g_loss_dev, nullptr,
             teacher_ids_dev, teacher_logits_dev, K, dlogits_out_dev, ld_out, status_dev};
  return cu(dtype ? launch_grad<__nv_bfloat16, 8>(distill_grad_kernel<__nv_bfloat16, 8>, a, st) : launch_grad<float, 8>(distill_grad_kernel<float, 8>, a, st));
}

size_t fv_linear_logprobs_workspace_bytes(int32_t rows, int32_t V) {
  if (rows <= 0 || V <= 0) return 0;
  return align_up((size_t)rows * V * 4, 256);
}

fv_status fv_linear_logprobs(const void* a_dev, const void* w_dev, const void* bias_dev, int32_t rows, int32_t C, int32_t V, float tau, const int32_t* ids_dev,
                             float* logprob_out_dev, float* stats_out_dev, float* entropy_out_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                             void* stream) {
  if (!workspace_dev || !al(workspace_dev, 256)) return FV_ERR_INVALID_ARG;
  if (workspace_bytes < fv_linear_logprobs_workspace_bytes(rows, V)) return FV_ERR_CAPACITY;
  const fv_status s = fv_gemm_bf16(a_dev, w_dev, bias_dev, rows, V, C, EPI_F32, workspace_dev, nullptr, nullptr, 0, rows, status_dev, nullptr, 0, stream);
  if (s != FV_OK) return s;
  return fv_token_logprobs(workspace_dev, 0, V, rows, V, tau, ids_dev, 0, logprob_out_dev, stats_out_dev, entropy_out_dev, nullptr, nullptr, status_dev, stream);
}

}  // extern "C"
