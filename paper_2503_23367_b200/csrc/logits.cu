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
#include <cstdlib>
#include <type_traits>

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
__device__ __forceinline__ float warp_max(float v) {   // (no NaN comes here)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// Untiled copy global -> this CTA's shared memory, its bytes counted on `bar`.  Both addresses and the size are multiples of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
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
// vector that are not the row's are -inf, which no pass notices.  The cluster's CTAs split the vectors evenly.  Thread t reads the
// vectors t, t + G, ... of its part.
template <typename T, int G> struct Slice {
  static constexpr int E = Elem<T>::E;
  const T* row;      // first logit of the row
  int off, V;        // elements between the 16-byte boundary and the row; logits of the row
  int v0, n, t;      // first vector of this part, their number; thread of the group
  int head, tail;    // this part's vectors that hold elements in front of or behind the row, or -1
  uint4* s;          // [n]
  __device__ __forceinline__ Slice(const T* row_, int V_, int rank, int lg_parts, int t_, uint4* s_) : row(row_), V(V_), t(t_), s(s_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    const int nv = (off + V + E - 1) / E, base = nv >> lg_parts, rem = nv & ((1 << lg_parts) - 1);
    n = base + (rank < rem);
    v0 = rank * base + min(rank, rem);
    head = v0 == 0 && off > 0 ? 0 : -1;
    tail = v0 + n == nv && (off + V) % E ? n - 1 : -1;
  }
  __device__ __forceinline__ int first_index(int v) const { return (v0 + v) * E - off; }   // index in the row of the vector's first element
  __device__ __forceinline__ bool whole(int v) const { return v != head && v != tail; }
  __device__ __forceinline__ void build(int v) {
    T* d = reinterpret_cast<T*>(s + v);
    const int i0 = first_index(v);
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = Elem<T>::load(row + min(max(i0 + e, 0), V - 1));   // all on their way before the first is stored
#pragma unroll
    for (int e = 0; e < E; ++e) Elem<T>::store(d + e, i0 + e >= 0 && i0 + e < V ? x[e] : -INFINITY);
  }
  // One copy for all whole vectors, completed on `bar`; the partial ones are built by the threads that hold them.
  __device__ __forceinline__ void fetch(uint64_t* bar) {
    if (t == 0) {
      const int lo = head == 0, hi = tail >= 0 ? max(n - 1, lo) : n;
      const uint32_t bytes = (uint32_t)(hi - lo) * 16;
      mbar_expect_tx(bar, bytes);
      if (bytes) bulk_load(smem_u32(s + lo), reinterpret_cast<const char*>(row - off) + (size_t)(v0 + lo) * 16, bytes, bar);
    }
    if (t == 0 && head == 0) build(0);
    if (tail >= 0 && tail != head && tail % G == t) build(tail);
  }
  // f(vector) for the thread's vectors, four loads at a time.
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const uint4* q = s + t;
    int left = n - t;
    for (; left > 3 * G; left -= 4 * G, q += 4 * G) {
      const uint4 a = q[0], b = q[G], c = q[2 * G], d = q[3 * G];
      f(a); f(b); f(c); f(d);
    }
    for (; left > 0; left -= G, q += G) f(*q);
  }
};

template <int G> __device__ __forceinline__ void group_sync() {
  if constexpr (G == 32) __syncwarp();
  else __syncthreads();
}

// Sums with the maximum known: s = sum e, t = sum e d, e = 2^d, d = (x - m) log2(e) / tau = (x - m) c.
//   Near: d is taken as x c - mc in one operation, mc = m c rounded.  That rounding (the slip, known exactly from another fused operation) moves all
//   exponents of the row alike, so sums can be put right at the end, and it is small where |m c| is; that saves half an instruction per
//   logit.  Rows farther from 0 (or masked with -1e9, or with the type's lowest value) take the difference first.
constexpr float kNear = 4096.f;        // |m c| below which the slip is below 2^-12
struct Sums { float s, t; };
template <bool NEAR> struct Expo {
  uint64_t a, b;
  __device__ __forceinline__ Expo(float m, float c) : a(pack2(c, c)), b(NEAR ? pack2(-(m * c), -(m * c)) : pack2(-m, -m)) {}
  __device__ __forceinline__ uint64_t operator()(uint64_t x) const { return NEAR ? fma2(x, a, b) : mul2(add2(x, b), a); }
  static __device__ __forceinline__ float slip(float m, float c) { return NEAR ? fmaf(m, c, -(m * c)) : 0.f; }   // d comes out too large by this
};
__device__ __forceinline__ uint64_t exp2_pair(uint64_t d) {
  float a, b;
  unpack2(d, a, b);
  return pack2(exp2_fast(a), exp2_fast(b));
}
template <typename T, int G, bool ENT, bool NEAR> __device__ __forceinline__ Sums thread_sums(const Slice<T, G>& sl, float m, float c) {
  constexpr int P = Elem<T>::E / 2;
  const Expo<NEAR> ex(m, c);
  uint64_t s[2] = {0, 0}, t[2] = {0, 0};
  sl.each([&](const uint4& u) {
    uint64_t x[P];
    Elem<T>::unpack(u, x);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t d = ex(x[i]), e = exp2_pair(d);
      s[i & 1] = add2(s[i & 1], e);
      if (ENT) t[i & 1] = fma2(e, d, t[i & 1]);
    }
  });
  Sums r{0.f, 0.f};
  float a, b;
  unpack2(add2(s[0], s[1]), a, b);
  r.s = a + b;
  if (ENT) {
    unpack2(add2(t[0], t[1]), a, b);
    r.t = a + b;
    if (r.t != r.t && r.s == r.s) {     // 0 * -inf: the thread has met logits of -inf, which add nothing
      t[0] = 0;
      sl.each([&](const uint4& u) {
        uint64_t x[P];
        Elem<T>::unpack(u, x);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const uint64_t d = ex(x[i]);
          unpack2(d, a, b);
          t[0] = fma2(exp2_pair(d), pack2(fmaxf(a, -1e30f), fmaxf(b, -1e30f)), t[0]);
        }
      });
      unpack2(t[0], a, b);
      r.t = a + b;
    }
  }
  return r;
}
__device__ __forceinline__ bool is_near(float m, float c) { return fabsf(m * c) < kNear; }

// What the parts of a row know of it, and what the whole row comes to.
struct Part { float m, s, t; };
struct Stat { float m, L, H, s; };
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }
template <bool ENT> __device__ __forceinline__ Stat stat_of(float m, float s, float t) {
  Stat r{m, logf(s), 0.f, s};
  if (ENT && s != 0.f) r.H = r.L - kLn2 * (t / s);
  return r;
}
// The whole row from its parts (at most 8), by a whole warp: a part's exponents were taken against its own maximum.
template <bool ENT> __device__ __forceinline__ Stat stat_of_parts(const Part* parts, int n, float c, int lane) {
  Part p{-INFINITY, 0.f, 0.f};
  if (lane < n) p = parts[lane];
  const float m = warp_max(p.m);
  const float up = (safe_max(p.m) - safe_max(m)) * c, f = p.s == 0.f ? 0.f : exp2_fast(up);   // s = 0: nothing but -inf, its up means nothing
  float s = p.s * f, t = ENT && f != 0.f ? fmaf(p.s, up, p.t) * f : 0.f;
#pragma unroll
  for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (ENT) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
  }
  s = __shfl_sync(0xFFFFFFFFu, s, 0);
  if (ENT) t = __shfl_sync(0xFFFFFFFFu, t, 0);
  return stat_of<ENT>(m, s, t);
}

// The row's copy has arrived.  A wait that runs out is reported; it is waited for once more, so that no copy lands after the kernel.
__device__ __forceinline__ void row_wait(uint64_t* bar, int32_t* status) {
  if (mbar_wait(bar, 0)) return;
  put_status(status, DEV_TIMEOUT_TMA);
  mbar_wait(bar, 0);
}

// ---- scratch of a group beside its slice ---------------------------------------------------------------------------------
constexpr int kFewAlt = 24;        // up to here the alternatives are bounded by the maxima of 32 groups of threads, beyond by those of 128
constexpr int kThreadGroups = 128;
template <int G, bool ALT> struct alignas(16) Scratch {
  static constexpr int kCand = !ALT ? 0 : G == 32 ? 256 : 1024;
  float gm[ALT && G > 32 ? kThreadGroups : 4];
  float2 red[G / 32];
  float red_m[G / 32];
  float m, thr;
  int count;
  unsigned long long bar;
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
    if ((sl.t & 31) == 0) sc.red_m[sl.t >> 5] = m;
    __syncthreads();
    m = sc.red_m[0];
#pragma unroll
    for (int w = 1; w < G / 32; ++w) m = fmaxf(m, sc.red_m[w]);
  }
  return m;
}
// The warp's values in descending order of the lanes (a bitonic network).
__device__ __forceinline__ float sort_descending(float v, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      const float o = __shfl_xor_sync(0xFFFFFFFFu, v, j);
      v = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(v, o) : fminf(v, o);
    }
  return v;
}
// The maximum, and a value that at least n_alt of the part's elements reach: the n_alt-th largest among the maxima of groups of threads.  Where large
// values are spread over the row, 1.2 n_alt elements reach that of 128 groups at n_alt 64, 1.8 n_alt that of 32 at 24 (of 24 at 24: 3.8 n_alt).  kLowest where fewer
// groups have a value.
template <typename T, int G> __device__ __forceinline__ float part_max_and_threshold(const Slice<T, G>& sl, Scratch<G, true>& sc, float mine, int n_alt, float& thr) {
  float m;
  const int lane = sl.t & 31;
  if (G == 32 || n_alt <= kFewAlt) {
    float g = mine;
    if constexpr (G > 32) {
      constexpr int SG = G / 32;
#pragma unroll
      for (int o = SG / 2; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
      if (sl.t % SG == 0) sc.gm[sl.t / SG] = g;
      __syncthreads();
      g = sc.gm[lane];
    }
    g = sort_descending(g, lane);
    m = __shfl_sync(0xFFFFFFFFu, g, 0);
    thr = __shfl_sync(0xFFFFFFFFu, g, n_alt - 1);
  } else if constexpr (G > 32) {
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

// The sums of the group's part against m, in every thread.
template <bool ENT, typename T, int G, bool ALT> __device__ __forceinline__ Sums part_sums(const Slice<T, G>& sl, Scratch<G, ALT>& sc, float m, float c) {
  const bool near = is_near(m, c);
  Sums r = near ? thread_sums<T, G, ENT, true>(sl, m, c) : thread_sums<T, G, ENT, false>(sl, m, c);
  r.s = warp_sum(r.s);
  if (ENT) r.t = warp_sum(r.t);
  if constexpr (G > 32) {
    if ((sl.t & 31) == 0) sc.red[sl.t >> 5] = make_float2(r.s, r.t);
    __syncthreads();
    r = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < G / 32; ++w) { r.s += sc.red[w].x; r.t += sc.red[w].y; }
  } else {
    __syncwarp();
  }
  if (near) {
    const float slip = Expo<true>::slip(m, c), f = fmaf(-kLn2, slip, 1.f);   // 2^-slip
    if (ENT) r.t = fmaf(-slip, r.s, r.t) * f;
    r.s *= f;
  }
  return r;
}

template <typename T> __device__ __forceinline__ float slice_elem(const uint4* s, int v, int e) {
  if constexpr (sizeof(T) == 4) return reinterpret_cast<const float*>(s + v)[e];
  else return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(s + v)[e]);
}

// The keys of the part's elements that reach the threshold, in any order.  Few threads hold one; a warp goes over the vectors of each such thread together.
template <typename T, int G> __device__ __forceinline__ void part_candidates(const Slice<T, G>& sl, Scratch<G, true>& sc, float mine, float thr) {
  const int lane = sl.t & 31;
  for (uint32_t who = __ballot_sync(0xFFFFFFFFu, mine >= thr); who; who &= who - 1) {
    for (int v = (sl.t & ~31) + __ffs(who) - 1 + lane * G; v < sl.n; v += 32 * G) {
      const uint4 u = sl.s[v];
      uint64_t x[Elem<T>::E / 2];
      Elem<T>::unpack(u, x);
      const int i0 = sl.first_index(v);
#pragma unroll
      for (int e = 0; e < Elem<T>::E; ++e) {
        float a, b;
        unpack2(x[e >> 1], a, b);
        const float f = e & 1 ? b : a;
        if (f >= thr) {
          const int slot = atomicAdd(&sc.count, 1);
          if (slot < Scratch<G, true>::kCand) sc.cand[slot] = alt_key(f, i0 + e);
        }
      }
    }
  }
  group_sync<G>();
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
  const void* x; long long ld; int rows, V, per_max, lg;   // per_max: vectors of the largest slice; lg: of the CTAs that share a row, the logarithm
  float inv_tau;
  const int32_t* ids; int n_alt;
  float* logprob; float2* stats; float* entropy; int32_t* alt_ids; float* alt_logprob;
  int32_t* status;
};

constexpr int kWarpRows = 2;       // rows of a CTA where a warp takes one
template <int G> constexpr int cta_threads() { return G == 32 ? 32 * kWarpRows : G; }
template <typename S> __host__ __device__ constexpr size_t group_bytes(int per_max) { return (size_t)per_max * 16 + sizeof(S); }

template <typename T, int G, bool ENT, bool ALT>
__global__ void __launch_bounds__(cta_threads<G>()) token_logprobs_kernel(const RowsArgs p) {
  using S = Scratch<G, ALT>;
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = G == 32 ? 1 : 1 << p.lg, rank = G == 32 ? 0 : (int)cluster_ctarank();
  const int sub = G == 32 ? threadIdx.x >> 5 : 0, t = G == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int row = G == 32 ? blockIdx.x * kWarpRows + sub : blockIdx.x >> p.lg;
  pdl_wait();
  if (G == 32 && row >= p.rows) return;
  if (G > 32 && parts > 1) cluster_arrive_relaxed();
  uint4* mine = reinterpret_cast<uint4*>(reinterpret_cast<char*>(smem) + sub * group_bytes<S>(p.per_max));
  S& sc = *reinterpret_cast<S*>(mine + p.per_max);
  const T* xrow = static_cast<const T*>(p.x) + row * p.ld;
  Slice<T, G> sl(xrow, p.V, rank, G == 32 ? 0 : p.lg, t, mine);
  uint64_t* bar = reinterpret_cast<uint64_t*>(&sc.bar);
  if (t == 0) { mbar_init(bar, 1); mbar_fence_init(); }
  if (ALT) {
    if (t < kMaxAlt) sc.list[t] = 0;
    if (G == 32) sc.list[t + 32] = 0;
    if (t == 0) sc.count = 0;
  }
  group_sync<G>();
  sl.fetch(bar);
  float xid = 0.f;
  int id = -1;
  if (t == 0 && rank == 0 && p.ids) {
    id = dep_load(p.ids + row);
    if (id >= 0 && id < p.V) xid = Elem<T>::load(xrow + id);
  }
  row_wait(bar, p.status);
  typename Elem<T>::Max mx;
  sl.each([&](const uint4& u) { mx.add(u); });
  const float own = mx.value(), c = p.inv_tau * kLog2e;
  float m, thr = 0.f;
  if constexpr (ALT) m = part_max_and_threshold<T, G>(sl, sc, own, p.n_alt, thr);
  else m = part_max<T, G, ALT>(sl, sc, own);
  const Sums tot = part_sums<ENT>(sl, sc, safe_max(m), c);
  if constexpr (ALT) {
    part_candidates<T, G>(sl, sc, own, thr);
    part_list<T, G>(sl, sc, p.n_alt);
  }
  const Part part{m, tot.s, tot.t};
  Stat st;
  unsigned long long* alts = sc.list;
  if (G == 32 || parts == 1) {
    st = stat_of<ENT>(m, tot.s, tot.t);
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
    st = stat_of_parts<ENT>(sc.part, parts, c, t & 31);
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
  const void* x; long long ld; int rows, V, per_max, lg;
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
      if (32 * i >= K) continue;
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
    for (int i = 0; i < P; ++i) {
      lq[i] = q[i] = 0.f;
      if (32 * i >= K) continue;
      lq[i] = (x[i] - m) * inv_tau;
      q[i] = expf(lq[i]);
      s += q[i];
    }
    s = warp_sum(s);
    some = __any_sync(0xFFFFFFFFu, any);
    bad = __any_sync(0xFFFFFFFFu, wrong);
    const float ls = logf(s);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (32 * i >= K) continue;
      q[i] = some ? q[i] / s : 0.f;
      lq[i] -= ls;
    }
  }
};
struct alignas(16) TeacherRow {    // of one row, for the gradient's corrections
  int id[kMaxTeacher];
  float q[kMaxTeacher], x[kMaxTeacher];
  int some;
};
// What entry k, which has a token, takes off its probability: all entries of that token together, at the first of them; -1 elsewhere.
__device__ __forceinline__ float teacher_share(const TeacherRow& tr, int k, int K) {
  const int id = tr.id[k];
  float sum = 0.f;
  bool first = true;
  for (int j = 0; j < K; j += 4) {         // (behind K: id -1)
    const int4 o = *reinterpret_cast<const int4*>(tr.id + j);
    const float4 q = *reinterpret_cast<const float4*>(tr.q + j);
    if (o.x == id) { sum += q.x; first &= j >= k; }
    if (o.y == id) { sum += q.y; first &= j + 1 >= k; }
    if (o.z == id) { sum += q.z; first &= j + 2 >= k; }
    if (o.w == id) { sum += q.w; first &= j + 3 >= k; }
  }
  return first ? sum : -1.f;
}

template <typename T> __device__ __forceinline__ bool same_alignment(const T* a, const T* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// f of every pair of logits of the part, written where the row's gradient lies.
template <typename T, int G, typename F> __device__ __forceinline__ void write_row(const Slice<T, G>& sl, T* drow, F f) {
  constexpr int E = Elem<T>::E, P = E / 2;
  const bool vec = same_alignment(sl.row, static_cast<const T*>(drow));
  T* dvec = drow - sl.off + (size_t)sl.v0 * E;
#pragma unroll 4
  for (int v = sl.t; v < sl.n; v += G) {
    uint64_t d[P];
    Elem<T>::unpack(sl.s[v], d);
#pragma unroll
    for (int i = 0; i < P; ++i) d[i] = f(d[i]);
    if (vec && sl.whole(v)) {
      *reinterpret_cast<uint4*>(dvec + (size_t)v * E) = Elem<T>::pack(d);
    } else {
      const int i0 = sl.first_index(v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float a, b;
        unpack2(d[e >> 1], a, b);
        if (i0 + e >= 0 && i0 + e < sl.V) Elem<T>::store(drow + i0 + e, e & 1 ? b : a);
      }
    }
  }
}

template <int G> struct alignas(16) DistillScratch { Scratch<G, false> sc; TeacherRow tr; };

template <typename T, int G, bool GRAD>
__global__ void __launch_bounds__(cta_threads<G>()) distill_kernel(const DistillArgs p) {
  using S = DistillScratch<G>;
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = G == 32 ? 1 : 1 << p.lg, rank = G == 32 ? 0 : (int)cluster_ctarank();
  const int sub = G == 32 ? threadIdx.x >> 5 : 0, t = G == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int row = G == 32 ? blockIdx.x * kWarpRows + sub : blockIdx.x >> p.lg;
  pdl_wait();
  if (G == 32 && row >= p.rows) return;
  if (G > 32 && parts > 1) cluster_arrive_relaxed();
  uint4* mine = reinterpret_cast<uint4*>(reinterpret_cast<char*>(smem) + sub * group_bytes<S>(p.per_max));
  S& own = *reinterpret_cast<S*>(mine + p.per_max);
  Scratch<G, false>& sc = own.sc;
  TeacherRow& tr = own.tr;
  const T* xrow = static_cast<const T*>(p.x) + row * p.ld;
  Slice<T, G> sl(xrow, p.V, rank, G == 32 ? 0 : p.lg, t, mine);
  uint64_t* bar = reinterpret_cast<uint64_t*>(&sc.bar);
  if (t == 0) { mbar_init(bar, 1); mbar_fence_init(); }
  group_sync<G>();
  sl.fetch(bar);
  Teacher te;
  float xk[Teacher::P];
  if (t < 32 && (GRAD || rank == 0)) {
    te.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, p.V, p.inv_tau, t);
#pragma unroll
    for (int i = 0; i < Teacher::P; ++i) {
      xk[i] = 0.f;
      if (GRAD || 32 * i < p.K) xk[i] = te.id[i] >= 0 ? Elem<T>::load(xrow + te.id[i]) : 0.f;
      if (GRAD) { tr.id[t + 32 * i] = te.id[i]; tr.q[t + 32 * i] = te.q[i]; tr.x[t + 32 * i] = xk[i]; }
    }
    if (GRAD && t == 0) tr.some = te.some;
  }
  row_wait(bar, p.status);
  typename Elem<T>::Max mx;
  sl.each([&](const uint4& u) { mx.add(u); });
  const float m = part_max<T, G, false>(sl, sc, mx.value()), c = p.inv_tau * kLog2e;
  const Sums tot = part_sums<false>(sl, sc, safe_max(m), c);
  const Part part{m, tot.s, 0.f};
  Stat st;
  if (G == 32 || parts == 1) {
    st = stat_of<false>(m, tot.s, 0.f);
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
    st = stat_of_parts<false>(sc.part, parts, c, t & 31);
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
    constexpr int E = Elem<T>::E;
    T* drow = static_cast<T*>(p.dx) + row * p.ld_dx;
    const float w = (p.g ? dep_load(p.g + row) : 1.f) * p.inv_tau;
    const bool none = !tr.some || w == 0.f || st.L == -INFINITY;   // (tr: written before the barriers of the sums)
    const bool near = is_near(st.m, c);
    const float f = none ? 0.f : near ? w / st.s * fmaf(-kLn2, Expo<true>::slip(st.m, c), 1.f) : w / st.s;
    if (none) write_row<T, G>(sl, drow, [&](uint64_t) { return uint64_t(0); });
    else if (near) write_row<T, G>(sl, drow, [&, ex = Expo<true>(st.m, c), f2 = pack2(f, f)](uint64_t x) { return mul2(exp2_pair(ex(x)), f2); });
    else write_row<T, G>(sl, drow, [&, ex = Expo<false>(st.m, c), f2 = pack2(f, f)](uint64_t x) { return mul2(exp2_pair(ex(x)), f2); });
    group_sync<G>();
    if (!none)
      for (int k = t; k < p.K; k += G) {
        const int id = tr.id[k];
        const int at = id < 0 ? -1 : (id + sl.off) / E - sl.v0;
        if (at < 0 || at >= sl.n) continue;
        const float share = teacher_share(tr, k, p.K);
        if (share < 0.f) continue;
        Elem<T>::store(drow + id, w * (exp2_fast((tr.x[k] - st.m) * c) / st.s - share));
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
        for (int e = 0; e < E; e += 2)
          f[e / 2] = pack2(Elem<T>::load(row + min(max(i0 + e, 0), V - 1)), Elem<T>::load(row + min(max(i0 + e + 1, 0), V - 1)));
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
  const int from = seg * 32 * U * E - sg.off, lo = max(0, from), hi = min(p.V, from + 32 * U * E);   // the logits of this warp
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

// Who takes a row: a warp, or a cluster of CTAs of 128 or 256 threads.
struct Shape { int group, lg, per_max; };
constexpr int kMaxRowBytes = 1536 << 10;
static int envi(const char* n, int d) { const char* s = getenv(n); return s ? atoi(s) : d; }
Shape row_shape(const void* x, long long ld, int rows, int V, int es, bool warp_may) {
  const int E = 16 / es;
  const bool aligned = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (ld * es) % 16 == 0;   // every row starts on a boundary
  const int nv = aligned ? (V + E - 1) / E : logits_vectors(V, E);
  static const int WV = envi("FV_WV", 1024), G1 = envi("FV_G1", 128), N1 = envi("FV_N1", 2048), SL = envi("FV_SL", 48), WR = envi("FV_WR", 8), LM = envi("FV_LM", 512);
  if (warp_may && nv <= WV && rows >= 148 * WR) return {32, 0, nv};
  int lg = 0;
  while ((1 << lg) < kMaxCluster && (size_t)((nv + (1 << lg) - 1) >> lg) * 16 > ((size_t)SL << 10)) ++lg;
  while ((1 << lg) < kMaxCluster && ((long long)rows << lg) < 148 && (nv >> (lg + 1)) >= LM) ++lg;
  const int per = (nv + (1 << lg) - 1) >> lg;
  return {per <= N1 ? G1 : 256, lg, per};
}

constexpr int kMaxSmem = 227 << 10;
template <typename K> cudaError_t allow_smem(K kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem); }
template <typename T> cudaError_t allow_all() {
  cudaError_t e = cudaSuccess;
  auto add = [&](auto kernel) { if (e == cudaSuccess) e = allow_smem(kernel); };
  auto group = [&](auto g) {
    constexpr int G = decltype(g)::value;
    add(token_logprobs_kernel<T, G, false, false>); add(token_logprobs_kernel<T, G, false, true>);
    add(token_logprobs_kernel<T, G, true, false>); add(token_logprobs_kernel<T, G, true, true>);
    add(distill_kernel<T, G, false>); add(distill_kernel<T, G, true>);
  };
  group(std::integral_constant<int, 32>()); group(std::integral_constant<int, 128>()); group(std::integral_constant<int, 256>());
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

template <typename F> cudaError_t with_group(int group, F f) {
  if (group == 32) return f(std::integral_constant<int, 32>());
  return group == 128 ? f(std::integral_constant<int, 128>()) : f(std::integral_constant<int, 256>());
}
template <int G, typename K, typename A> cudaError_t go_rows(K kernel, const A& a, size_t bytes, cudaStream_t st) {   // bytes: of a group's shared memory
  const unsigned grid = G == 32 ? (a.rows + kWarpRows - 1) / kWarpRows : (unsigned)a.rows << a.lg;
  return launch_clusters(kernel, grid, cta_threads<G>(), 1 << a.lg, bytes * (G == 32 ? kWarpRows : 1), st, a);
}
template <typename T> cudaError_t launch_token(RowsArgs& a, cudaStream_t st) {
  const Shape s = row_shape(a.x, a.ld, a.rows, a.V, sizeof(T), a.n_alt <= kFewAlt);
  a.per_max = s.per_max; a.lg = s.lg;
  return with_group(s.group, [&](auto g) {
    constexpr int G = decltype(g)::value;
    const size_t with = group_bytes<Scratch<G, true>>(s.per_max), without = group_bytes<Scratch<G, false>>(s.per_max);
    if (a.n_alt > 0) return a.entropy ? go_rows<G>(token_logprobs_kernel<T, G, true, true>, a, with, st) : go_rows<G>(token_logprobs_kernel<T, G, false, true>, a, with, st);
    return a.entropy ? go_rows<G>(token_logprobs_kernel<T, G, true, false>, a, without, st) : go_rows<G>(token_logprobs_kernel<T, G, false, false>, a, without, st);
  });
}
template <typename T> cudaError_t launch_distill(DistillArgs& a, cudaStream_t st) {
  const Shape s = row_shape(a.x, a.ld, a.rows, a.V, sizeof(T), true);
  a.per_max = s.per_max; a.lg = s.lg;
  return with_group(s.group, [&](auto g) {
    constexpr int G = decltype(g)::value;
    const size_t bytes = group_bytes<DistillScratch<G>>(s.per_max);
    return a.dx ? go_rows<G>(distill_kernel<T, G, true>, a, bytes, st) : go_rows<G>(distill_kernel<T, G, false>, a, bytes, st);
  });
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
  RowsArgs a{logits_dev, ld, rows, V, 0, 0, 1.f / tau, ids_dev, n_alt, logprob_out_dev, reinterpret_cast<float2*>(stats_out_dev), entropy_out_dev,
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
  DistillArgs a{logits_dev, ld, rows, V, 0, 0, 1.f / tau, teacher_ids_dev, teacher_logits_dev, K, g_loss_dev, loss_out_dev, reinterpret_cast<float2*>(stats_out_dev),
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
