// Rows of logits: log probabilities of given tokens with entropy and top alternatives, distillation from a teacher's top
// logits, and the gradients of both.  For a row x of V logits at temperature tau
//     m = max_j x_j,  d_j = (x_j - m) / tau,  s = sum_j exp(d_j),  L = ln s,  p_j = exp(d_j - L)
//     logprob(id) = d_id - L,     H = L - sum_j exp(d_j) d_j / s
//     d logprob / dx_j = (1[j = id] - p_j) / tau,     dH / dx_j = -p_j (ln p_j + H) / tau
//     loss = sum_k q_k (ln q_k - ln p_{id_k}),  q = softmax(t / tau),     d loss / dx_j = (p_j - sum_{k: id_k = j} q_k) / tau
// Everything here does a handful of operations per logit, so DRAM bounds it where there is work enough, and in the smallest calls the chain of
// dependent steps.  Three forms, by what has to be known of a row before it can be left:
//   statistics, alternatives, the loss alone: rows stream through the registers once (Stream, token_logprobs_kernel, distill_loss_kernel);
//   the loss with its gradient: rows stay in shared memory between the sums and the gradient (Slice, distill_kernel);
//   gradients from known statistics: a warp per 128 or 256 vectors of a row, no shared memory (Segment, *_grad_kernel).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <cstdint>
#include <type_traits>

#include "internal.h"
#include "logits.cuh"
#include "sm100.cuh"   // the device status codes, cluster barriers

namespace fv {

using namespace logits_detail;

namespace {

constexpr int kMaxAlt = 64;        // alternatives of a row
constexpr int kMaxTeacher = 128;   // entries of a teacher's row
constexpr int kMaxCluster = 8;     // CTAs that share a row
// Read once: first to leave the caches (and, like dep_load16, it stays where it is written).
__device__ __forceinline__ uint4 load16_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_smem(const void* p, uint32_t cta) {   // the same shared-memory address in another CTA of the cluster
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(cta));
  return r;
}
__device__ __forceinline__ void peer_store(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ void peer_store(uint32_t addr, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void peer_store(uint32_t addr, uint64_t v) { asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory"); }
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
// vector that are not the row's are -inf, which no pass notices.  The cluster's CTAs split the vectors evenly.  Thread t copies and reads the
// vectors t, t + G, ... of its part, so it needs no barrier before its own passes.
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
  __device__ __forceinline__ void fetch() const {
    const char* g = reinterpret_cast<const char*>(row - off) + (size_t)(v0 + t) * 16;
    const uint32_t d = smem_u32(s + t);
    const int left = n - t;
#pragma unroll 4
    for (int i = 0; i < left; i += G)
      if (whole(t + i)) cp_async16(d + i * 16, g + (size_t)i * 16);
    if (t == 0 && head == 0) build(0);
    if (tail >= 0 && tail != head && tail % G == t) build(tail);
  }
  __device__ __forceinline__ void build(int v) const {   // a vector that is the row's in part
    T* d = reinterpret_cast<T*>(s + v);
    const int i0 = first_index(v);
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = Elem<T>::load(row + min(max(i0 + e, 0), V - 1));   // all on their way before the first is stored
#pragma unroll
    for (int e = 0; e < E; ++e) Elem<T>::store(d + e, i0 + e >= 0 && i0 + e < V ? x[e] : -INFINITY);
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

// s = sum e and t = sum e d over vectors of logits.
template <typename T, bool ENT> struct Sums {
  uint64_t s[2] = {0, 0}, t[2] = {0, 0};
  template <typename X> __device__ __forceinline__ void add(const uint4& u, const X& ex) {
    constexpr int P = Elem<T>::E / 2;
    uint64_t x[P];
    Elem<T>::unpack(u, x);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t d = ex(x[i]), e = exp2_pair(d);
      s[i & 1] = add2(s[i & 1], e);
      if (ENT) {
        float a, b;
        unpack2(d, a, b);
        t[i & 1] = fma2(e, pack2(fmaxf(a, -1e30f), fmaxf(b, -1e30f)), t[i & 1]);   // a logit of -inf adds 0, not 0 * -inf
      }
    }
  }
};

// The whole row from its parts, one of each warp that went over it (at most 64), by a whole warp.
template <bool ENT> __device__ __forceinline__ Stat stat_of_parts(const Part* parts, int n, float c, int lane) {
  Part p{-INFINITY, 0.f, 0.f};
  if (lane < n) p = {parts[lane].m, parts[lane].s, ENT ? parts[lane].t : 0.f};
  if (n > 32) {
    Part q{-INFINITY, 0.f, 0.f};
    if (lane + 32 < n) q = {parts[lane + 32].m, parts[lane + 32].s, ENT ? parts[lane + 32].t : 0.f};
    const float m = fmaxf(p.m, q.m);
    p = against<ENT>(p, m, c);
    q = against<ENT>(q, m, c);
    p.s += q.s;
    p.t += q.t;
  }
  p = warp_union<ENT>(p, c);
  return stat_of<ENT>(p.m, p.s, p.t);
}

struct RowsArgs {
  const void* x; long long ld; int rows, V;
  int per_max, lg;    // vectors of the largest part of a row; log2 of the CTAs that share one
  float inv_tau;
  int32_t* status;
};

// ---- rows that are read once: a stream through the registers ---------------------------------------------------------------
// A warp (G 32) or the four warps of a CTA (G 128; in a cluster each CTA has a part of the row) go over a row.  Thread t reads the whole
// vectors t, t + G, ... of its part, in blocks of four, and keeps a running maximum beside sums against a reference that changes only where
// the maximum passes it by 2^kRise.  The blocks come through a ring in shared memory in which every lane has its own slots: copies of
// kAhead blocks are on their way while one is summed, which in registers would cost half of the warps.  Nothing of the row is kept; what holds
// the alternatives is read again, from L2.
constexpr int kStreamThreads = 128, kStreamWarps = 4, kBlock = 4, kAhead = 1;
constexpr int kRingBytes = (kAhead + 1) * kBlock * 32 * 16;   // of a warp
constexpr int kMaxWarps = kMaxCluster * kStreamWarps;   // warps that share a row

template <typename T, int G> struct Stream {
  static constexpr int E = Elem<T>::E, B = kBlock;
  const T* row;      // first logit of the row
  int off, V, v0;    // elements between the 16-byte boundary and the row; logits of the row; first vector of this part
  int t, nw, part;   // thread of the group; whole vectors of the part; the partial vector that this thread has beside, or -1
  const char* base;  // the part's first whole vector
  __device__ __forceinline__ Stream(const T* row_, int V_, int rank, int lg_parts, int t_) : row(row_), V(V_), t(t_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    const int nv = (off + V + E - 1) / E, b = nv >> lg_parts, rem = nv & ((1 << lg_parts) - 1);
    const int n = b + (rank < rem), v = rank * b + min(rank, rem);
    const bool head = v == 0 && off > 0 && n > 0, tail = n > 0 && v + n == nv && (off + V) % E && !(head && n == 1);
    part = head && t == 0 ? 0 : tail && t == G - 1 ? nv - 1 : -1;
    v0 = v + head;
    nw = n - head - tail;
    base = reinterpret_cast<const char*>(row - off) + (size_t)v0 * 16;
  }
  __device__ __forceinline__ int turns() const { return (nw + B * G - 1) / (B * G); }   // blocks of the thread that has most
  __device__ __forceinline__ uint4 load(int j) const { return dep_load16(base + (size_t)j * 16); }
  __device__ __forceinline__ int index_of(int j) const { return (v0 + j) * E - off; }   // logit that whole vector j starts with
  __device__ __forceinline__ uint4 partial() const {            // its elements that are not the row's are -inf
    float x[E];
    const int i0 = part * E - off;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = Elem<T>::load(row + min(max(i0 + e, 0), V - 1));
    uint64_t f[E / 2];
#pragma unroll
    for (int e = 0; e < E; e += 2)
      f[e / 2] = pack2(i0 + e >= 0 && i0 + e < V ? x[e] : -INFINITY, i0 + e + 1 >= 0 && i0 + e + 1 < V ? x[e + 1] : -INFINITY);
    return Elem<T>::pack(f);
  }
  // f(vectors, how many, block) for the thread's blocks of up to B vectors (32 apart in the ring), the partial one last and alone (block -1).  ring: the warp's.
  template <typename F> __device__ __forceinline__ void each(uint4* ring, F f) const {
    const uint32_t slot = smem_u32(ring + (t & 31));
    const char* g = base + (size_t)t * 16;
    int left = nw - t, next = left;              // vectors times G that are not summed, not asked for
    const auto ask = [&](int s) {
#pragma unroll
      for (int i = 0; i < B; ++i)
        if (next > i * G) cp_async16(slot + (s * B + i) * 512, g + (size_t)i * G * 16);
      asm volatile("cp.async.commit_group;" ::: "memory");
      next -= B * G;
      g += (size_t)B * G * 16;
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) ask(s);
    int k = 0;
    for (int s = 0; left > 0; ++k, left -= B * G, s = s == kAhead ? 0 : s + 1) {
      ask(s == 0 ? kAhead : s - 1);              // into the block before this one, which the lane has read
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
      const uint4* mine = ring + s * B * 32 + (t & 31);
      if (left > (B - 1) * G) {
        f(mine, std::integral_constant<int, B>(), k);
      } else {
        for (int i = 0; left > i * G; ++i) f(mine + i * 32, std::integral_constant<int, 1>(), k);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (part >= 0) {
      const uint4 a = partial();
      f(&a, std::integral_constant<int, 1>(), -1);
    }
  }
};

// The running state of a thread.  Exponents reach kRise before the reference follows, and t then holds up to kRise s, whose roundings stay in the entropy.  Where the largest logit stands more than 2^kRise above what its
// thread met before, it becomes the reference, so the entropy of a nearly certain row keeps the digits of the plain sum (largest error over rows of 4096, 20011 and 131072 whose entropy is 1e-9 ... 0.7: 6e-7, the
// plain fp32 form's 9e-7; with a rise of 64 and whole references 8e-6).  Against a rise of 64 it costs nothing on rows of a spread of 2.5 and at most 1.5 % on rows of a spread of 8 (8192 x 4096 fp32 26.5 -> 26.9 us); 4 has
// the same errors.
constexpr float kRise = 8.f;
template <typename T, bool ENT> struct Online {
  float c, m = -INFINITY, R = 0.f, limit = -INFINITY;   // limit: largest maximum that the reference bears
  Sums<T, ENT> sums;
  __device__ __forceinline__ explicit Online(float c_) : c(c_) {}
  template <int N> __device__ __forceinline__ float add(const uint4* u) {   // u: N vectors of the ring, 32 apart; their maximum
    typename Elem<T>::Max mx;
#pragma unroll
    for (int i = 0; i < N; ++i) mx.add(u[i * 32]);
    const float bm = mx.value();
    m = fmaxf(m, bm);
    if (bm > limit) {
      const float to = reference(bm, c);
      if (limit != -INFINITY) {
        const float d = R - to, f = exp2_fast(d);
        const uint64_t d2 = pack2(d, d), f2 = pack2(f, f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (ENT) sums.t[i] = mul2(fma2(sums.s[i], d2, sums.t[i]), f2);
          sums.s[i] = mul2(sums.s[i], f2);
        }
      }
      R = to;
      limit = bm + kRise / c;
    }
    const Expo<true> ex(R, c);
#pragma unroll
    for (int i = 0; i < N; ++i) sums.add(u[i * 32], ex);
    return bm;
  }
  __device__ __forceinline__ Part part() const { return part_of(m, sums, delta(safe_max(m), c, R)); }
};
// A row whose maximum m is far from 0: the sums once more, against it.
template <typename T, int G, bool ENT> __device__ __forceinline__ Part far_part(const Stream<T, G>& st, uint4* ring, float m, float c) {
  Sums<T, ENT> sums;
  const Expo<false> ex(m, c);
  st.each(ring, [&](const uint4* u, auto n, int) {
#pragma unroll
    for (int i = 0; i < decltype(n)::value; ++i) sums.add(u[i * 32], ex);
  });
  return part_of(m, sums, 0.f);
}

// ---- alternatives --------------------------------------------------------------------------------------------------------
constexpr int kFewAlt = 24;        // up to here they are bounded by the maxima of 32 groups of threads, beyond by those of 128
constexpr int kThreadGroups = 128;
constexpr int kMaxCand = 256;      // elements that a warp can keep
struct alignas(16) WarpAlt {
  unsigned long long cand[kMaxCand];
  float gm[32];
  uint16_t hit[kMaxCand];
};
static_assert(sizeof(WarpAlt) <= kRingBytes, "takes the ring's place");
struct alignas(16) RowAlt {        // of a row that warps share (in every CTA of a cluster)
  float own[kThreadGroups], all[kThreadGroups];   // maxima of groups of threads, of this CTA and of the cluster
  float bound[kMaxCluster];        // what the cluster's CTAs found on their own
  float least[kStreamWarps];
  int count[kMaxWarps];            // of the warps' lists, which lie behind this: [warps][n_alt], in the cluster's first CTA
};

__device__ __forceinline__ int larger_than(float my, const float* gm, int n) {   // how many of gm are
  int count = 0;
#pragma unroll 8
  for (int j = 0; j < n; j += 4) {
    const float4 v = *reinterpret_cast<const float4*>(gm + j);
    count += (v.x > my) + (v.y > my) + (v.z > my) + (v.w > my);
  }
  return count;
}
__device__ __forceinline__ float warp_min(float v) {
  float r;
  asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// The n-th largest of the maxima of 32 groups of threads, which is the smallest that fewer than n exceed: at least n of the elements that the groups went over
// reach it, about n (1 + n / 40) where large values are spread over them.  Every warp for itself.
__device__ __forceinline__ float nth_of_32(const float* gm, int n, int lane) {
  const float my = gm[lane];
  return warp_min(larger_than(my, gm, 32) < n ? my : INFINITY);
}
// The same of 128 groups (1.2 n elements at n 64), by the CTA.  least: [4] of the CTA's own.
__device__ __forceinline__ float nth_of_128(const float* gm, float* least, int n) {
  const float my = gm[threadIdx.x];
  const float w = warp_min(larger_than(my, gm, kThreadGroups) < n ? my : INFINITY);
  if ((threadIdx.x & 31) == 0) least[threadIdx.x >> 5] = w;
  __syncthreads();
  const float r = fminf(fminf(least[0], least[1]), fminf(least[2], least[3]));
  __syncthreads();
  return r;
}
// The largest of v over groups of 32 / per neighbouring lanes (per a power of two), in each of their lanes.
__device__ __forceinline__ float lane_group_max(float v, int per) {
  for (int o = 16 / per; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}

// What a warp has found: keys in no order, all of them larger than what it has left out.
struct Found {
  unsigned long long* key;   // [kMaxCand]
  int n, lane;
  unsigned long long floor;  // smallest key worth keeping
  // Every lane brings some elements of a vector (a bit each).  False where they do not fit.
  template <typename T> __device__ __forceinline__ bool add(const uint4& u, uint32_t bits, int index) {
    for (uint32_t who; (who = __ballot_sync(0xFFFFFFFFu, bits != 0)) != 0;) {
      if (n + __popc(who) > kMaxCand) return false;
      if (bits) {
        const int e = __ffs(bits) - 1;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        uint32_t word = w[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) word = (sizeof(T) == 4 ? e : e >> 1) == i ? w[i] : word;
        const float f = sizeof(T) == 4 ? __uint_as_float(word) : __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16);
        key[n + __popc(who & ((1u << lane) - 1))] = alt_key(f, index + e);
        bits &= bits - 1;
      }
      n += __popc(who);
    }
    return true;
  }
  // Down to the `most` largest, in descending order.
  __device__ __forceinline__ void cut(int most) {
    __syncwarp();
    unsigned long long k[kMaxCand / 32];
    int place[kMaxCand / 32];
#pragma unroll
    for (int i = 0; i < kMaxCand / 32; ++i) {
      place[i] = kMaxCand;
      if (32 * i >= n) continue;
      k[i] = lane + 32 * i < n ? key[lane + 32 * i] : 0;
      if (lane + 32 * i < n) place[i] = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) place[i] += key[j] > k[i];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kMaxCand / 32; ++i)
      if (place[i] < most) key[place[i]] = k[i];
    __syncwarp();
    n = min(n, most);
    if (n == most) floor = key[n - 1] + 1;
  }
};
template <typename T> __device__ __forceinline__ uint32_t reach_bits(const uint4& u, float thr) {   // elements of at least thr
  constexpr int E = Elem<T>::E;
  typename Elem<T>::Max mx;
  mx.add(u);
  if (!(mx.value() >= thr)) return 0;
  uint64_t x[E / 2];
  Elem<T>::unpack(u, x);
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    float a, b;
    unpack2(x[e / 2], a, b);
    bits |= (a >= thr ? 1u << e : 0u) | (b >= thr ? 2u << e : 0u);
  }
  return bits;
}

// The warp's elements that reach thr, at most `most` of them where there are many.  bm: [turns][32] maxima of the lanes' blocks.  A few blocks hold one: their vectors
// are read again, spread over the warp.  Where they are too many (rows of mostly equal values, rows in order), the warp goes over all of its
// vectors once more and keeps the largest `most` of what it has met whenever it runs out of room.
template <typename T, int G> __device__ __forceinline__ void warp_select(const Stream<T, G>& st, const T* bm, float partial_max, float thr, int most, WarpAlt& wa, Found& f) {
  constexpr int B = Stream<T, G>::B;
  const int lane = st.t & 31, turns = st.turns();
  const uint32_t below = (1u << lane) - 1;
  f.key = wa.cand;
  f.lane = lane;
  f.n = 0;
  f.floor = 1;
  uint4 u{};
  const uint32_t mine = st.part >= 0 && partial_max >= thr;
  if (__any_sync(0xFFFFFFFFu, mine)) {
    if (mine) u = st.partial();
    f.add<T>(u, mine ? reach_bits<T>(u, thr) : 0, st.part * Elem<T>::E - st.off);
  }
  int h = 0;
  for (int k0 = 0; k0 < turns; k0 += 4) {
    float b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = k0 + i < turns ? float(bm[(k0 + i) * 32 + lane]) : -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool hit = b[i] >= thr;
      const uint32_t who = __ballot_sync(0xFFFFFFFFu, hit);
      if (!who) continue;
      const int at = h + __popc(who & below);
      if (hit && at < kMaxCand) wa.hit[at] = (uint16_t)((k0 + i) * 32 + lane);
      h += __popc(who);
    }
  }
  __syncwarp();
  bool fits = h <= kMaxCand;
  const int t0 = st.t - lane;
  for (int q0 = 0; fits && q0 < B * h; q0 += 128) {
    uint4 v[4];
    int j[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = q0 + 32 * i + lane;
      j[i] = st.nw;
      if (q0 + 32 * i >= B * h) continue;
      if (q < B * h) {
        const int code = wa.hit[q / B];
        j[i] = t0 + (code & 31) + ((code >> 5) * B + q % B) * G;
      }
      if (j[i] < st.nw) v[i] = st.load(j[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (fits && q0 + 32 * i < B * h) fits = f.add<T>(v[i], j[i] < st.nw ? reach_bits<T>(v[i], thr) : 0, st.index_of(j[i]));
  }
  if (fits) {
    __syncwarp();
    return;
  }
  f.n = 0;
  const auto over = [&](const uint4& x, uint32_t bits, int index) {
    uint32_t rest = bits;
    while (__any_sync(0xFFFFFFFFu, rest != 0)) {       // one element of each lane at a time
      const uint32_t low = rest & -rest;
      if (f.n > kMaxCand - 32) f.cut(most);
      uint32_t take = low;
      if (low) {                                       // what is below the kept ones is left out
        const int e = __ffs(low) - 1;
        uint64_t p[Elem<T>::E / 2];
        Elem<T>::unpack(x, p);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < Elem<T>::E; ++i) {
          float a, b;
          unpack2(p[i / 2], a, b);
          if (i == e) v = i & 1 ? b : a;
        }
        if (alt_key(v, index + e) < f.floor) take = 0;
      }
      f.add<T>(x, take, index);
      rest &= ~low;
    }
  };
  if (__any_sync(0xFFFFFFFFu, mine)) over(u, mine ? reach_bits<T>(u, thr) : 0, st.part * Elem<T>::E - st.off);
  for (int q = 0; q < turns * B; ++q) {
    if (!__any_sync(0xFFFFFFFFu, float(bm[q / B * 32 + lane]) >= thr)) continue;
    const int j = st.t + q * G;
    uint4 x{};
    if (j < st.nw) x = st.load(j);
    over(x, j < st.nw ? reach_bits<T>(x, thr) : 0, st.index_of(j));
  }
  f.cut(most);
}

// ---- log probabilities of given tokens, statistics, entropy, alternatives ------------------------------------------------
struct TokenArgs {
  RowsArgs r;
  const int32_t* ids; int n_alt, turns;     // turns: blocks of the thread that has most
  float* logprob; float2* stats; float* entropy; int32_t* alt_ids; float* alt_logprob;
};
// The scratch of a row that warps share: what each of them has found, and what it finds where the row has to be gone over again.
struct alignas(16) Shared { Part part[2][kMaxWarps]; };
// Every CTA of the cluster has every warp's part, behind a barrier of all threads that share the row.
template <bool ENT> __device__ __forceinline__ void share_parts(Shared& sh, const Part& part, int turn, int parts, int rank, int warp, int lane) {
  if (lane < parts) {
    const uint32_t to = peer_smem(&sh.part[turn][rank * kStreamWarps + warp], lane);
    peer_store(to, part.m); peer_store(to + 4, part.s);
    if (ENT) peer_store(to + 8, part.t);
  }
  __syncwarp();
  if (parts > 1) cluster_sync_all();
  else __syncthreads();
}

template <bool ENT> __device__ __forceinline__ void tell_alt(const TokenArgs& p, int row, const Stat& st, int place, unsigned long long key) {   // key 0: none
  const bool bad = st.L != st.L;
  p.alt_ids[(size_t)row * p.n_alt + place] = bad || !key ? -1 : alt_index(key);
  p.alt_logprob[(size_t)row * p.n_alt + place] = bad ? st.L : key ? (alt_value(key) - st.m) * p.r.inv_tau - st.L : -INFINITY;
}
template <typename T, bool ENT> __device__ __forceinline__ void tell_row(const TokenArgs& p, int row, const Stat& st, int id, float xid) {
  if (p.stats) p.stats[row] = make_float2(st.m, st.L);
  if (ENT) p.entropy[row] = st.H;
  if (!p.logprob) return;
  float lp = 0.f;                      // -1: the row has no token
  if (id >= 0 && id < p.r.V) {
    lp = st.L == -INFINITY ? -INFINITY : (xid - st.m) * p.r.inv_tau - st.L;
  } else if (id != -1) {
    put_status(p.r.status, DEV_BAD_TOKEN_ID);
    lp = __int_as_float(0x7FC00000);
  }
  p.logprob[row] = lp;
}

// One read of the rows.  Counted per 32 logits of rows of 50021: 5.9 warp instructions (bf16; fp32 6.4) with one exponential per logit, 1.6 more with the entropy; and per
// row, with alternatives, 740 more for a warp's (4096, 8 of them) or 4500 for four warps' (50021, 20 of them).  So long rows are bound by DRAM (4800 x 32768 fp32 93 us, 6.8 TB/s with what L2 held) or, bf16 with entropy and alternatives, by
// instructions (3001 x 50021, 20 alternatives, 69 us, issue 67 %); many short rows by how many are on their way beside the 6700 clocks behind each one's last logit (8192 x 4096
// fp32, 8 alternatives, 27 us, 4.9 TB/s); few rows by the chain of steps (two of 4096 with 5 alternatives 4.2 us, four of 131072 with 20 on clusters of eight 6.9).
template <typename T, int G, bool ENT, bool ALT>
__global__ void __launch_bounds__(kStreamThreads, 8) token_logprobs_kernel(const TokenArgs p) {
  constexpr int W = kStreamWarps;
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = G == 32 ? 1 : 1 << p.r.lg, rank = parts > 1 ? (int)cluster_ctarank() : 0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = G == 32 ? blockIdx.x * W + warp : blockIdx.x >> p.r.lg;
  if (parts > 1) cluster_arrive_relaxed();
  pdl_wait();
  if (G == 32 && row >= p.r.rows) return;
  // shared memory: per warp a ring, whose place the scratch of the alternatives takes later, and its block maxima; what warps share and their lists of alternatives
  const size_t per_warp = kRingBytes + (ALT ? (size_t)p.turns * 32 * sizeof(T) : 0);
  uint4* ring = reinterpret_cast<uint4*>(reinterpret_cast<char*>(smem) + warp * per_warp);
  WarpAlt& wa = *reinterpret_cast<WarpAlt*>(ring);
  T* bm = reinterpret_cast<T*>(reinterpret_cast<char*>(ring) + kRingBytes);   // (a maximum of Ts is a T)
  Shared& sh = *reinterpret_cast<Shared*>(reinterpret_cast<char*>(smem) + W * per_warp);
  RowAlt& ra = *reinterpret_cast<RowAlt*>(&sh + 1);
  unsigned long long* lists = reinterpret_cast<unsigned long long*>(&ra + 1);   // [warps][n_alt]
  const T* xrow = static_cast<const T*>(p.r.x) + row * p.r.ld;
  const bool scribe = (G == 32 ? lane : threadIdx.x) == 0 && rank == 0;       // writes the row's numbers
  int id = -1;
  if (scribe && p.ids) id = dep_load(p.ids + row);
  const Stream<T, G> st(xrow, p.r.V, rank, G == 32 ? 0 : p.r.lg, G == 32 ? lane : threadIdx.x);
  const float c = p.r.inv_tau * kLog2e;
  Online<T, ENT> on(c);
  float partial_max = -INFINITY;
  if (ALT)                             // the thread's last block, which may be short, and those that it does not have
    for (int k = (st.t < st.nw ? (st.nw - st.t + G - 1) / G : 0) / Stream<T, G>::B; k < st.turns(); ++k) Elem<T>::store(bm + k * 32 + lane, -INFINITY);
  st.each(ring, [&](const uint4* u, auto n, int k) {
    const float b = on.template add<decltype(n)::value>(u);
    if (ALT) {
      if (k < 0) partial_max = b;
      else Elem<T>::store(bm + k * 32 + lane, decltype(n)::value > 1 ? b : fmaxf(float(bm[k * 32 + lane]), b));
    }
  });
  float xid = 0.f;
  if (id >= 0 && id < p.r.V) xid = Elem<T>::load(xrow + id);
  Part mine = on.part();
  if constexpr (G == 32) {
    const float m = warp_max(mine.m);
    if (!is_near(safe_max(m), c)) mine = far_part<T, G, ENT>(st, ring, m, c);
    const Part all = warp_union<ENT>(mine, c);
    const Stat stat = stat_of<ENT>(all.m, all.s, all.t);
    if constexpr (ALT) {
      wa.gm[lane] = on.m;
      __syncwarp();
      const float thr = fmaxf(nth_of_32(wa.gm, p.n_alt, lane), Elem<T>::kLowest);   // -inf is no alternative
      Found f;
      warp_select(st, bm, partial_max, thr, p.n_alt, wa, f);
      for (int i = lane; i < max(f.n, p.n_alt); i += 32) {    // every key's place is how many are larger
        int place = i;
        unsigned long long key = 0;
        if (i < f.n) {
          key = f.key[i];
          place = 0;
#pragma unroll 4
          for (int j = 0; j < f.n; ++j) place += f.key[j] > key;
        }
        if (place < p.n_alt) tell_alt<ENT>(p, row, stat, place, key);
      }
    }
    if (scribe) tell_row<T, ENT>(p, row, stat, id, xid);
  } else {
    __syncwarp();
    if (parts > 1) cluster_wait();     // every CTA of the cluster has started
    if constexpr (ALT) {
      // What every alternative reaches: the bound of this CTA's thread groups; in a cluster the largest of its CTAs' bounds, or that of
      // groups over all of them.  The first holds where the large values lie in one part of the row, the second where they are spread.
      const bool few = p.n_alt <= kFewAlt;
      const int per = few ? 32 / W : kThreadGroups / W;        // groups of a warp
      const float g = lane_group_max(on.m, per);
      if (lane % (32 / per) == 0) ra.own[warp * per + lane / (32 / per)] = g;
      __syncthreads();
      float thr = few ? nth_of_32(ra.own, p.n_alt, lane) : nth_of_128(ra.own, ra.least, p.n_alt);
      if (parts > 1) {
        const int gw = per >> p.r.lg;                          // groups of a warp where the cluster has 32 or 128 (at least one: 8 CTAs have 32 warps)
        const float h = lane_group_max(on.m, gw);
        const int i = lane >> p.r.lg;
        const float v = __shfl_sync(0xFFFFFFFFu, h, i * (32 / gw) & 31);
        if (i < gw) peer_store(peer_smem(&ra.all[(rank * W + warp) * gw + i], lane & (parts - 1)), v);
        if ((int)threadIdx.x < parts) peer_store(peer_smem(&ra.bound[rank], threadIdx.x), thr);
        __syncwarp();
        cluster_sync_all();
        for (int i = 0; i < parts; ++i) thr = fmaxf(thr, ra.bound[i]);
        thr = fmaxf(thr, few ? nth_of_32(ra.all, p.n_alt, lane) : nth_of_128(ra.all, ra.least, p.n_alt));
      }
      thr = fmaxf(thr, Elem<T>::kLowest);                      // -inf is no alternative
      Found f;
      warp_select(st, bm, partial_max, thr, p.n_alt, wa, f);
      if (f.n > p.n_alt) f.cut(p.n_alt);
      unsigned long long* list = lists + (size_t)(rank * W + warp) * p.n_alt;
      for (int i = lane; i < f.n; i += 32) peer_store(peer_smem(list + i, 0), (uint64_t)f.key[i]);
      if (lane == 0) peer_store(peer_smem(&ra.count[rank * W + warp], 0), f.n);
    }
    share_parts<ENT>(sh, warp_union<ENT>(mine, c), 0, parts, rank, warp, lane);
    const int warps = parts * W;
    const float m = warp_max(lane < warps ? sh.part[0][lane].m : -INFINITY);
    const bool near = is_near(safe_max(m), c);
    if (!near) share_parts<ENT>(sh, warp_union<ENT>(far_part<T, G, ENT>(st, ring, m, c), c), 1, parts, rank, warp, lane);
    if (rank != 0 || (!ALT && warp != 0)) return;
    const Stat stat = stat_of_parts<ENT>(sh.part[near ? 0 : 1], warps, c, lane);
    if constexpr (ALT) {               // the lists one behind the other, in a ring's place; then every key's place is how many are larger
      const int per = kStreamThreads / warps, l = threadIdx.x / per;   // threads of a list; this thread's
      const int have = lane < warps ? ra.count[lane] : 0;
      int upto = have;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += v;
      }
      const int total = __shfl_sync(0xFFFFFFFFu, upto, 31), from = __shfl_sync(0xFFFFFFFFu, upto - have, l), n = __shfl_sync(0xFFFFFFFFu, have, l);
      unsigned long long* all = reinterpret_cast<unsigned long long*>(smem);
      static_assert((size_t)kMaxWarps * kMaxAlt * 8 + 16 <= W * ((size_t)kRingBytes + 32 * sizeof(T)), "32 lists of 64 keys and one more fit the rings and block maxima");
      for (int i = threadIdx.x % per; i < n; i += per) all[from + i] = lists[(size_t)l * p.n_alt + i];
      if (threadIdx.x == 0) all[total] = 0;                      // (keys are read in pairs)
      __syncthreads();
      for (int i = threadIdx.x; i < max(total, p.n_alt); i += kStreamThreads) {
        unsigned long long key = 0;
        int place = i;
        if (i < total) {
          key = all[i];
          place = 0;
#pragma unroll 4
          for (int j = 0; j < total; j += 2) {
            const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(all + j);
            place += (k.x > key) + (k.y > key);
          }
        }
        if (place < p.n_alt) tell_alt<ENT>(p, row, stat, place, key);
      }
    }
    if (scribe) tell_row<T, ENT>(p, row, stat, id, xid);
  }
}

// ---- distillation: loss, and with GRAD its gradient while the row is still in shared memory --------------------------------
struct DistillArgs {
  RowsArgs r;
  const int32_t* t_ids; const float* t_logits; int K;
  const float* g;                  // [rows] or null: 1
  float* loss; float2* stats;
  void* dx; long long ld_dx;
};

// The teacher's row: lane l of one warp holds the entries l, l + 32, ...; q over the entries that have a token (-1: none), lq = ln q.
struct TeacherEntries {
  static constexpr int P = kMaxTeacher / 32;
  int id[P];
  float x[P];
  __device__ __forceinline__ void load(const int32_t* ids, const float* logits, int K, int lane) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      id[i] = -1;
      x[i] = -INFINITY;
      if (lane + 32 * i < K) { id[i] = dep_load(ids + lane + 32 * i); x[i] = dep_load(logits + lane + 32 * i); }
    }
  }
};
struct Teacher {
  static constexpr int P = TeacherEntries::P;
  int id[P];
  float q[P], lq[P];
  bool some, bad;
  __device__ __forceinline__ void weigh(const TeacherEntries& e, int K, int V, float inv_tau) {
    float x[P], m = -INFINITY;
    bool wrong = false, any = false;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const bool has = e.id[i] >= 0 && e.id[i] < V;
      wrong |= !has && e.id[i] != -1;
      id[i] = has ? e.id[i] : -1;
      x[i] = has ? e.x[i] : -INFINITY;
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
    const float ls = logf(s), inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (32 * i >= K) continue;
      q[i] = some ? q[i] * inv : 0.f;
      lq[i] -= ls;
    }
  }
};
struct alignas(16) TeacherRow {    // the same in shared memory; behind K: id -1
  int id[kMaxTeacher];
  float q[kMaxTeacher];
  int some;                       // whether it has an entry
  __device__ __forceinline__ void put(const Teacher& te, int lane) {
#pragma unroll
    for (int i = 0; i < Teacher::P; ++i) { id[lane + 32 * i] = te.id[i]; q[lane + 32 * i] = te.q[i]; }
  }
};
// What an entry takes off its token's probability: q, where no token comes twice; else all entries of the token together, at the first of them, -1 at the
// others.  tr holds what te does.
__device__ __forceinline__ void teacher_shares(const Teacher& te, const TeacherRow& tr, int K, int lane, float (&share)[Teacher::P]) {
  constexpr int P = Teacher::P;
  bool twice = false;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    share[i] = te.id[i] >= 0 ? te.q[i] : -1.f;
    if (32 * i >= K) continue;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, te.id[i]);
    twice |= te.id[i] >= 0 && (same & (same - 1)) != 0;
#pragma unroll
    for (int j = 0; j < i; ++j)
#pragma unroll 8
      for (int r = 0; r < 32; ++r) {
        const int other = __shfl_sync(0xFFFFFFFFu, te.id[j], (lane + r) & 31);   // (by every lane)
        twice |= te.id[i] >= 0 && te.id[i] == other;
      }
  }
  if (!__any_sync(0xFFFFFFFFu, twice)) return;
  for (int i = 0; i < P; ++i) {
    const int k = lane + 32 * i, id = tr.id[k];
    float sum = 0.f;
    bool first = id >= 0;
    for (int j = 0; j < K; ++j) {
      if (tr.id[j] != id) continue;
      sum += tr.q[j];
      first &= j >= k;
    }
    const float s = first ? sum : -1.f;
#pragma unroll
    for (int n = 0; n < P; ++n) share[n] = n == i ? s : share[n];
  }
}

// The row's loss and statistics, by the warp that has the teacher's entries; x: the logits of their tokens.
__device__ __forceinline__ void tell_loss(const DistillArgs& p, int row, const Teacher& te, const float (&x)[Teacher::P], const Stat& st, int lane) {
  float loss = 0.f;
#pragma unroll
  for (int i = 0; i < Teacher::P; ++i) {
    const float lp = st.L == -INFINITY ? -INFINITY : (x[i] - st.m) * p.r.inv_tau - st.L;
    if (te.id[i] >= 0 && te.q[i] != 0.f) loss = fmaf(te.q[i], te.lq[i] - lp, loss);   // (q NaN: the loss too)
  }
  loss = warp_sum(loss);
  if (lane != 0) return;
  if (te.bad) { put_status(p.r.status, DEV_BAD_TOKEN_ID); loss = __int_as_float(0x7FC00000); }
  p.loss[row] = loss;
  if (p.stats) p.stats[row] = make_float2(st.m, st.L);
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
      __stcs(reinterpret_cast<uint4*>(dvec + (size_t)v * E), Elem<T>::pack(d));
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

// G threads go over the row; one more warp deals with the teacher meanwhile: it weighs the entries, reads their tokens' logits, adds up the entries of
// the same token, and at the end writes the loss and puts the gradient of those tokens right.
// What every thread finds in its vectors: their maximum, and the sums against it.  No barrier: the warps' results are put together once.
template <typename T, int G> __device__ __forceinline__ Part thread_part(const Slice<T, G>& sl, float c) {
  typename Elem<T>::Max mx;
  sl.each([&](const uint4& u) { mx.add(u); });
  const float m = mx.value(), m0 = safe_max(m);
  Sums<T, false> sums;
  if (__all_sync(0xFFFFFFFFu, is_near(m0, c))) {
    const float R = reference(m0, c);
    sl.each([&, ex = Expo<true>(R, c)](const uint4& u) { sums.add(u, ex); });
    return part_of(m, sums, delta(m0, c, R));
  }
  sl.each([&, ex = Expo<false>(m0, c)](const uint4& u) { sums.add(u, ex); });
  return part_of(m, sums, 0.f);
}

struct alignas(16) DistillScratch { Part part[64]; TeacherRow tr; };

// One read and one write of the rows, two exponentials per logit: 4096 x 131072 bf16 380 us, 5.7 TB/s with the exponentials' unit 67 % busy; 8192 x 4096 fp32 45 us, 5.9 TB/s.  The
// row could be read a second time from L2 instead of being kept; that is 1.5 times L2's traffic where L2 is the faster by less.
template <typename T, int G>
__global__ void __launch_bounds__(G + 32, G == 64 ? 10 : 768 / G) distill_kernel(const DistillArgs p) {
  constexpr int W = G / 32, E = Elem<T>::E, P = Teacher::P;
  extern __shared__ uint4 smem[];
  pdl_trigger();
  const int parts = 1 << p.r.lg, rank = parts > 1 ? (int)cluster_ctarank() : 0, t = threadIdx.x, warp = t >> 5, lane = t & 31, row = blockIdx.x >> p.r.lg;
  DistillScratch& sc = *reinterpret_cast<DistillScratch*>(smem + p.r.per_max);
  TeacherRow& tr = sc.tr;
  if (parts > 1) cluster_arrive_relaxed();
  pdl_wait();
  const float c = p.r.inv_tau * kLog2e;
  const T* xrow = static_cast<const T*>(p.r.x) + row * p.r.ld;
  T* drow = static_cast<T*>(p.dx) + row * p.ld_dx;
  const Slice<T, G> sl(xrow, p.r.V, rank, p.r.lg, t, smem);
  const float wg = (p.g ? dep_load(p.g + row) : 1.f) * p.r.inv_tau;
  // Two barriers: behind the first the parts are complete, the logits of the teacher's tokens read (in place they are overwritten next) and tr.some is
  // written; behind the second the row's gradient is written.
  if (warp < W) {
    sl.fetch();
    cp_async_wait_all();
    const Part part = warp_union<false>(thread_part(sl, c), c);
    __syncwarp();
    if (parts == 1) {
      if (lane == 0) sc.part[warp] = part;
      __syncthreads();
    } else {
      cluster_wait();                  // every CTA of the cluster has started
      if (lane < parts) {
        const uint32_t to = peer_smem(&sc.part[rank * W + warp], lane);
        peer_store(to, part.m); peer_store(to + 4, part.s); peer_store(to + 8, 0.f);
      }
      __syncwarp();
      cluster_sync_all();
    }
    const Stat st = stat_of_parts<false>(sc.part, parts * W, c, lane);
    if (!tr.some || wg == 0.f || st.L == -INFINITY) {
      write_row<T, G>(sl, drow, [](uint64_t) { return uint64_t(0); });
    } else if (is_near(st.m, c)) {
      const float R = reference(st.m, c), f = wg / st.s * exp2_fast(delta(st.m, c, R));
      write_row<T, G>(sl, drow, [ex = Expo<true>(R, c), f2 = pack2(f, f)](uint64_t x) { return mul2(exp2_pair(ex(x)), f2); });
    } else {
      const float f = wg / st.s;
      write_row<T, G>(sl, drow, [ex = Expo<false>(st.m, c), f2 = pack2(f, f)](uint64_t x) { return mul2(exp2_pair(ex(x)), f2); });
    }
    __syncthreads();
    return;
  }
  Teacher te;
  float x[P], share[P], keep = 0.f;
  TeacherEntries entries;
  entries.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, lane);
#pragma unroll
  for (int i = 0; i < P; ++i) x[i] = entries.id[i] >= 0 && entries.id[i] < p.r.V ? Elem<T>::load(xrow + entries.id[i]) : 0.f;
  te.weigh(entries, p.K, p.r.V, p.r.inv_tau);
  if (lane == 0) tr.some = te.some;
  tr.put(te, lane);
  __syncwarp();
  teacher_shares(te, tr, p.K, lane, share);
#pragma unroll
  for (int i = 0; i < P; ++i) keep += x[i];
  asm volatile("" ::"f"(keep) : "memory");   // the logits have arrived
  __syncwarp();
  if (parts > 1) { cluster_wait(); cluster_sync_all(); }
  else __syncthreads();
  const Stat st = stat_of_parts<false>(sc.part, parts * W, c, lane);
  if (rank == 0) tell_loss(p, row, te, x, st, lane);
  __syncthreads();
  if (te.some && wg != 0.f && st.L != -INFINITY) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int id = te.id[i], at = id < 0 ? -1 : (id + sl.off) / E - sl.v0;
      if (at >= 0 && at < sl.n && !(share[i] < 0.f)) Elem<T>::store(drow + id, wg * (exp2_fast((x[i] - st.m) * c) / st.s - share[i]));
    }
  }
}

// One read of the rows, then the teacher's entries (two dependent reads, some 150 instructions) by a warp: 1025 x 32768 bf16 15.6 us, 4.3 TB/s of one round of CTAs.
// The loss alone: nothing of the row is needed again but the logits of the teacher's tokens.
template <typename T, int G>
__global__ void __launch_bounds__(kStreamThreads, 8) distill_loss_kernel(const DistillArgs p) {
  constexpr int W = kStreamWarps;
  __shared__ Shared sh;
  __shared__ uint4 rings[W][kRingBytes / 16];
  pdl_trigger();
  const int parts = G == 32 ? 1 : 1 << p.r.lg, rank = parts > 1 ? (int)cluster_ctarank() : 0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = G == 32 ? blockIdx.x * W + warp : blockIdx.x >> p.r.lg;
  if (parts > 1) cluster_arrive_relaxed();
  pdl_wait();
  if (G == 32 && row >= p.r.rows) return;
  const T* xrow = static_cast<const T*>(p.r.x) + row * p.r.ld;
  const Stream<T, G> st(xrow, p.r.V, rank, G == 32 ? 0 : p.r.lg, G == 32 ? lane : threadIdx.x);
  uint4* ring = rings[warp];
  const float c = p.r.inv_tau * kLog2e;
  Online<T, false> on(c);
  st.each(ring, [&](const uint4* u, auto n, int) { on.template add<decltype(n)::value>(u); });
  Part mine = on.part();
  Stat stat;
  if constexpr (G == 32) {
    const float m = warp_max(mine.m);
    if (!is_near(safe_max(m), c)) mine = far_part<T, G, false>(st, ring, m, c);
    const Part all = warp_union<false>(mine, c);
    stat = stat_of<false>(all.m, all.s, all.t);
  } else {
    __syncwarp();
    if (parts > 1) cluster_wait();     // every CTA of the cluster has started
    share_parts<false>(sh, warp_union<false>(mine, c), 0, parts, rank, warp, lane);
    const float m = warp_max(lane < parts * W ? sh.part[0][lane].m : -INFINITY);
    const bool near = is_near(safe_max(m), c);
    if (!near) share_parts<false>(sh, warp_union<false>(far_part<T, G, false>(st, ring, m, c), c), 1, parts, rank, warp, lane);
    if (rank != 0 || warp != 0) return;
    stat = stat_of_parts<false>(sh.part[near ? 0 : 1], parts * W, c, lane);
  }
  TeacherEntries entries;
  entries.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, lane);
  float x[Teacher::P];
#pragma unroll
  for (int i = 0; i < Teacher::P; ++i) x[i] = entries.id[i] >= 0 && entries.id[i] < p.r.V ? Elem<T>::load(xrow + entries.id[i]) : 0.f;
  Teacher te;
  te.weigh(entries, p.K, p.r.V, p.r.inv_tau);
  tell_loss(p, row, te, x, stat, lane);
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
constexpr int kGradWarps = 4, kGradVectors = 4, kDistillGradVectors = 8;   // warps of a CTA; vectors of a lane

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
        x[u] = load16_once(row + i0);
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
      __stcs(reinterpret_cast<uint4*>(drow + i0), Elem<T>::pack(d));
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

// Bound by DRAM: 8192 x 4096 fp32 with entropy 42 us, 6.4 TB/s; 2003 x 50021 bf16 60 us, 6.7 TB/s (what stays in L2 at the end included).  U of 2 / 4 / 8: fp32 56 / 48 / 51 us
// before loads and stores were marked to leave the caches first, which is worth 6 us more.
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

// As above, and every warp weighs the teacher's entries itself (some 200 instructions beside 600 for its logits: U 8) and looks for tokens that come twice, which grows with the square of K / 32: 2048 x 16384 fp32, K 32:
// 46 us, 5.8 TB/s; K 128: 168.  4096 x 131072 bf16, K 64: 408 us, 5.3 TB/s; K 128: 701.
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
  TeacherEntries entries;
  entries.load(p.t_ids + (size_t)row * p.K, p.t_logits + (size_t)row * p.K, p.K, lane);
  Teacher te;
  te.weigh(entries, p.K, p.V, p.inv_tau);
  if (te.bad && seg == 0 && lane == 0) put_status(p.status, DEV_BAD_TOKEN_ID);
  const float m = dep_load(&p.stats[row].x), L = dep_load(&p.stats[row].y);
  const float w = (p.g_logprob ? dep_load(p.g_logprob + row) : 1.f) * p.inv_tau;
  if (!te.some || w == 0.f || L == -INFINITY) {
    sg.zero();
    return;
  }
  float xk[Teacher::P];
  tr.put(te, lane);
  const int from = seg * 32 * U * E - sg.off, lo = max(0, from), hi = min(p.V, from + 32 * U * E);   // the logits of this warp
#pragma unroll
  for (int i = 0; i < Teacher::P; ++i) {
    const int id = te.id[i];
    xk[i] = 0.f;
    if (id >= lo && id < hi) xk[i] = Elem<T>::load(xrow + id);
  }
  __syncwarp();                        // in place: read before any lane writes
  float share[Teacher::P];
  teacher_shares(te, tr, p.K, lane, share);
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
#pragma unroll
  for (int i = 0; i < Teacher::P; ++i) {
    const int id = te.id[i];
    if (id >= lo && id < hi && !(share[i] < 0.f)) Elem<T>::store(drow + id, w * (exp2_fast(fmaf(xk[i] - m, c, -L2)) - share[i]));
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
  cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Who takes a row.  Streamed: a warp, or a cluster of CTAs of 128 threads.  Kept in shared memory: a cluster of CTAs of 64, 128 or 256 threads.
struct Shape { int group, lg, per_max; };   // per_max: vectors of the largest part
constexpr int kMaxRowBytes = 1536 << 10;
int row_vectors(const void* x, long long ld, int V, int es) {
  const bool aligned = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (ld * es) % 16 == 0;   // every row starts on a boundary
  return aligned ? (V + 16 / es - 1) / (16 / es) : logits_vectors(V, 16 / es);
}
// CTAs that share a row, as a logarithm: as many as give every SM one, while a part has at least 1024 vectors (16 KB; below that the cluster's barriers cost what
// the shorter part saves: one row of 32 KB 2.5 us on one CTA, 2.3 on two; of 256 KB 8.2 on one, 2.8 on eight).
int spread(int nv, int rows, int lg) {
  while ((1 << lg) < kMaxCluster && ((long long)rows << lg) < 148 && (nv >> (lg + 1)) >= 1024) ++lg;
  return lg;
}
// A warp to a row where rows are short or so many that the warps fill the GPU: no barrier, a quarter of the instructions that a row takes beside its logits.
// us, a warp / a CTA of four, fp32, entropy alone and with 8 alternatives: 600 rows of 4 KB 2.2 / 3.0, 4.0 / 7.8; 1200 of 16 KB 5.7 / 4.7, 9.2 / 10.5; 4800 of 16 KB 9.3 / 13.1, 13.4 / 30.2;
// 4800 of 32 KB 27 / 26, 32 / 40; 2400 of 64 KB 32 / 27, 33 / 35; 2400 of 128 KB 58 / 51, 70 / 58.  More alternatives than a warp's 32 lanes can bound take the CTA.
Shape stream_shape(int nv, int rows, int n_alt) {
  if (n_alt <= kFewAlt && (nv <= 512 || (nv <= 1024 && rows >= 148 * 8) || (nv <= 2048 && rows >= 148 * 24))) return {32, 0, nv};
  const int lg = spread(nv, rows, 0);
  return {128, lg, (nv + (1 << lg) - 1) >> lg};
}
// Parts of at most 32 KB, six to an SM, for rows of up to 256 KB: us for 4096 rows of 256 KB, 64 threads to a part of up to 2048 vectors 455, 128 383, 256 568; parts of 64 KB and 256 threads 386.
// Longer rows stay with eight CTAs, whose parts grow to 192 KB: fewer to an SM.  us, loss and gradient in this one call / in two (fv_distill_topk, then fv_distill_topk_grad) / the bytes of one read and
// one write: 1024 x 131072 fp32 189 / 265 / 164, 1024 x 200000 fp32 304 / 406 / 251, bf16 199 / 216 / 125, 1024 x 393216 bf16 343 / 417 / 246; at the end of the range 256 x 390000 fp32 244 / 234 / 122.
Shape kept_shape(int nv, int rows) {
  int lg = 0;
  while ((1 << lg) < kMaxCluster && (nv + (1 << lg) - 1) >> lg > 2048) ++lg;
  lg = spread(nv, rows, lg);
  const int per = (nv + (1 << lg) - 1) >> lg;
  return {per <= 1024 ? 64 : per <= 2048 ? 128 : 256, lg, per};
}

constexpr int kMaxSmem = 227 << 10;
template <typename K> cudaError_t allow_smem(K kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem); }
template <typename T> cudaError_t allow_all() {
  cudaError_t e = cudaSuccess;
  auto add = [&](auto kernel) { if (e == cudaSuccess) e = allow_smem(kernel); };
  auto group = [&](auto g) {
    constexpr int G = decltype(g)::value;
    add(token_logprobs_kernel<T, G, false, true>); add(token_logprobs_kernel<T, G, true, true>);
  };
  group(std::integral_constant<int, 32>()); group(std::integral_constant<int, 128>());
  add(distill_kernel<T, 64>); add(distill_kernel<T, 128>); add(distill_kernel<T, 256>);
  return e;
}
// Function attributes belong to a device: set on the first call on each.
cudaError_t logits_init() {
  static std::atomic<uint64_t> done{0};
  return once_per_device(done, [] {
    const cudaError_t e = allow_all<float>();
    return e == cudaSuccess ? allow_all<__nv_bfloat16>() : e;
  });
}

template <typename K, typename A> cudaError_t go_rows(K kernel, int threads, A& a, const Shape& s, size_t smem, cudaStream_t st) {
  a.r.per_max = s.per_max; a.r.lg = s.lg;
  const unsigned grid = s.group == 32 ? (a.r.rows + kStreamWarps - 1) / kStreamWarps : (unsigned)a.r.rows << s.lg;
  return launch_clusters(kernel, grid, threads, 1 << s.lg, smem, st, a);
}
template <typename T, int G> cudaError_t go_token(TokenArgs& a, const Shape& s, cudaStream_t st) {
  a.turns = (s.per_max + Stream<T, G>::B * G - 1) / (Stream<T, G>::B * G);
  const size_t rows = kStreamWarps * (size_t)kRingBytes + (G == 32 ? 0 : sizeof(Shared));
  const size_t with = rows + kStreamWarps * (size_t)a.turns * 32 * sizeof(T) + (G == 32 ? 0 : sizeof(RowAlt) + ((size_t)a.n_alt * kStreamWarps * 8 << s.lg));
  if (a.n_alt > 0)
    return a.entropy ? go_rows(token_logprobs_kernel<T, G, true, true>, kStreamThreads, a, s, with, st) : go_rows(token_logprobs_kernel<T, G, false, true>, kStreamThreads, a, s, with, st);
  return a.entropy ? go_rows(token_logprobs_kernel<T, G, true, false>, kStreamThreads, a, s, rows, st) : go_rows(token_logprobs_kernel<T, G, false, false>, kStreamThreads, a, s, rows, st);
}
template <typename T> cudaError_t launch_token(TokenArgs& a, cudaStream_t st) {
  const Shape s = stream_shape(row_vectors(a.r.x, a.r.ld, a.r.V, sizeof(T)), a.r.rows, a.n_alt);
  return s.group == 32 ? go_token<T, 32>(a, s, st) : go_token<T, 128>(a, s, st);
}
template <typename T> cudaError_t launch_distill(DistillArgs& a, cudaStream_t st) {
  const int nv = row_vectors(a.r.x, a.r.ld, a.r.V, sizeof(T));
  if (!a.dx) {
    const Shape s = stream_shape(nv, a.r.rows, 0);
    return s.group == 32 ? go_rows(distill_loss_kernel<T, 32>, kStreamThreads, a, s, 0, st) : go_rows(distill_loss_kernel<T, 128>, kStreamThreads, a, s, 0, st);
  }
  const Shape s = kept_shape(nv, a.r.rows);
  const size_t smem = (size_t)s.per_max * 16 + sizeof(DistillScratch);
  if (s.group == 64) return go_rows(distill_kernel<T, 64>, 64 + 32, a, s, smem, st);
  return s.group == 128 ? go_rows(distill_kernel<T, 128>, 128 + 32, a, s, smem, st) : go_rows(distill_kernel<T, 256>, 256 + 32, a, s, smem, st);
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
  TokenArgs a{{logits_dev, ld, rows, V, 0, 0, 1.f / tau, status_dev}, ids_dev, n_alt, 0, logprob_out_dev, reinterpret_cast<float2*>(stats_out_dev), entropy_out_dev,
              alt_ids_out_dev, alt_logprob_out_dev};
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
  if (dtype) return cu(g_entropy_dev ? launch_grad<B, kGradVectors>(token_logprobs_grad_kernel<B, kGradVectors, true>, a, st) : launch_grad<B, kGradVectors>(token_logprobs_grad_kernel<B, kGradVectors, false>, a, st));
  return cu(g_entropy_dev ? launch_grad<float, kGradVectors>(token_logprobs_grad_kernel<float, kGradVectors, true>, a, st) : launch_grad<float, kGradVectors>(token_logprobs_grad_kernel<float, kGradVectors, false>, a, st));
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
  DistillArgs a{{logits_dev, ld, rows, V, 0, 0, 1.f / tau, status_dev}, teacher_ids_dev, teacher_logits_dev, K, g_loss_dev, loss_out_dev,
                reinterpret_cast<float2*>(stats_out_dev), dlogits_out_dev, ld_out};
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
  return cu(dtype ? launch_grad<__nv_bfloat16, kDistillGradVectors>(distill_grad_kernel<__nv_bfloat16, kDistillGradVectors>, a, st)
                  : launch_grad<float, kDistillGradVectors>(distill_grad_kernel<float, kDistillGradVectors>, a, st));
}

}  // extern "C"
