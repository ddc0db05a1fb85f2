// Log probabilities, statistics and entropy of the rows a * W^T + bias without their logits: the likelihood of tokens under the output head.
// With the logits stored, 8192 x 4096 of them cost 134 MB written and read again beside a product of 137 GFLOP; here a tile of the product stays in
// tensor memory until its columns have become, per row, a maximum and two sums (16 bytes per 128 columns).
//   The product is the CTA pair of gemm_pair.cu: 256 x BN tiles, tcgen05.mma.cta_group::2, operands by TMA, every wait bounded.
//   Sums: the tensor core cuts an accumulator's fp32 sum after every 16 products, which over 2048 of them shrinks a logit by 2e-6 of itself; so a tile is accumulated
//   in segments of kSegment of K, in turn in two accumulators, and the epilogue's threads add the segments in their registers, rounding to nearest
//   (8192 x 4096 x 2048: relative error of the statistics 2.2e-6 in one piece).  A thread has half a tile's columns of one row: eight warps with up to 128
//   accumulators per thread.  The additions and the exponentials of a tile run beside the next segments' products.
//   Then linear_finish_kernel puts the parts of a row together.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <type_traits>

#include "internal.h"
#include "logits.cuh"
#include "sm100.cuh"

namespace fv {

using namespace logits_detail;

namespace {

constexpr int BM = 128, BK = 64, KPS = 2;        // rows of a CTA; k of a block; blocks of a pipeline stage
constexpr int kATileBytes = BM * BK * 2;
constexpr int kSegment = 512;                    // k accumulated in one piece
constexpr int kSegmentBlocks = kSegment / BK;
constexpr int kEpilogueWarps = 8, kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kAccStride = 256, kTmemCols = 512;

template <int BN> struct Cfg {
  static constexpr int kSubBytes = kATileBytes + BN / 2 * BK * 2;   // one k-block: this CTA's rows of A, its half of the tile's rows of W
  static constexpr int kStageBytes = KPS * kSubBytes;
  static constexpr int kStages = BN == 256 ? 3 : 4;
  static constexpr int kSmem = kStages * kStageBytes + 256 /*barriers*/ + 1024 /*alignment slack*/;
};

struct LinearArgs {
  int M, N, K;
  float c;                          // log2(e) / tau
  const __nv_bfloat16* bias;
  const int32_t* ids;
  float4* part;                     // [2 * column tiles][M]: m, s, t of half a tile's columns of a row
  float* xid;                       // [M] logit of the row's token
  int32_t* status;
};

__device__ __forceinline__ float load_bf16(const __nv_bfloat16* p) {   // stays where it is written, like dep_load
  unsigned short v;
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
  return __uint_as_float((uint32_t)v << 16);
}

// acc[i] of a register array, i at run time: a tree of selections.
template <int N> __device__ __forceinline__ float pick(const float* acc, int i) {
  if constexpr (N == 1) {
    return acc[0];
  } else {
    const float lo = pick<N / 2>(acc, i), hi = pick<N / 2>(acc + N / 2, i);
    return i & (N / 2) ? hi : lo;
  }
}

// Bound by the product: 8192 x 2048 -> 4096 97 us, 1.42 PFLOP/s (the plain bf16 GEMM of the shape 92), the tensor pipe active 78 % of the SMs' time; a round of tiles ends with one epilogue that nothing
// covers (1.6 us), small calls are the fixed cost of a pair kernel (169 x 1024 -> 4096 9 us with the second launch: 32 tiles on 64 SMs).  320 threads leave 168 registers a thread, of which the 256-wide
// build spills 68 bytes (128 accumulators); the 128-wide one, 160 registers, none.
template <int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_logprobs_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const LinearArgs p) {
  using C = Cfg<BN>;
  constexpr int STAGES = C::kStages, COLS = BN / 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + STAGES * C::kStageBytes);   // used in the leader
  uint64_t* empty_bar = full_bar + STAGES;   // one per CTA, completed by the leader's commits
  uint64_t* acc_full = empty_bar + STAGES;   // [2] one per CTA
  uint64_t* acc_empty = acc_full + 2;        // [2] used in the leader: an arrival of every epilogue thread of the pair
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);

  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int tiles_m = (p.M + 2 * BM - 1) / (2 * BM), tiles_n = (p.N + BN - 1) / BN;
  const int total_tiles = tiles_m * tiles_n, num_kb = (p.K + BK - 1) / BK;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 2 * 32 * kEpilogueWarps); }
    mbar_fence_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  }
  cluster_sync_all();  // the peer's barriers exist before anything is signalled across the pair
  if (warp == 1) { tmem_alloc_pair(tmem_slot, kTmemCols); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      int pre = 0;  // stages of the first tile whose part of W is already on its way (W is a constant of the stream)
      if (pair < total_tiles) {
        const int n0 = (pair / tiles_m) * BN + (int)rank * (BN / 2);
        pre = min(STAGES, (num_kb + KPS - 1) / KPS);
        for (int i = 0; i < pre; ++i) {
          if (rank == 0) mbar_expect_tx(&full_bar[i], 2 * C::kStageBytes);
          for (int u = 0; u < KPS; ++u)   // (a k-block beyond K reads zeros)
            tma_load_2d_pair(smem + i * C::kStageBytes + u * C::kSubBytes + kATileBytes, &tmB, (KPS * i + u) * BK, n0, &full_bar[i]);
        }
      }
      pdl_wait();
      for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
        const int m0 = (tile % tiles_m) * (2 * BM) + (int)rank * BM, n0 = (tile / tiles_m) * BN + (int)rank * (BN / 2);
        for (int kb = 0; kb < num_kb; kb += KPS, ++it) {
          const int s = it % STAGES;
          uint8_t* a_s = smem + s * C::kStageBytes;
          if ((int)it < pre) {
            for (int u = 0; u < KPS; ++u) tma_load_2d_pair(a_s + u * C::kSubBytes, &tmA, (kb + u) * BK, m0, &full_bar[s]);
            continue;
          }
          if (!mbar_wait(&empty_bar[s], ((it / STAGES) & 1) ^ 1)) { put_status(p.status, DEV_TIMEOUT_TMA); ok = false; break; }
          if (rank == 0) mbar_expect_tx(&full_bar[s], 2 * C::kStageBytes);
          for (int u = 0; u < KPS; ++u) {
            tma_load_2d_pair(a_s + u * C::kSubBytes, &tmA, (kb + u) * BK, m0, &full_bar[s]);
            tma_load_2d_pair(a_s + u * C::kSubBytes + kATileBytes, &tmB, (kb + u) * BK, n0, &full_bar[s]);
          }
        }
      }
    }
  } else if (warp == 1) {
    pdl_wait();
    if (rank == 0) {
      constexpr uint32_t idesc = umma_idesc_bf16(2 * BM, BN);
      const bool leader = elect_one();
      uint32_t seg = 0, s = 0, ph = 0;   // segments so far; ring stage and its phase
      bool ok = true;
      for (int tile = pair; ok && tile < total_tiles; tile += npairs)
        for (int k0 = 0; ok && k0 < num_kb; k0 += kSegmentBlocks, ++seg) {
          const uint32_t buf = seg & 1;
          if (!mbar_wait(&acc_empty[buf], ((seg >> 1) & 1) ^ 1)) { put_status(p.status, DEV_TIMEOUT_MMA); ok = false; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + buf * kAccStride;
          const int k1 = min(num_kb, k0 + kSegmentBlocks);
          for (int kb = k0; kb < k1; kb += KPS) {
            if (!mbar_wait(&full_bar[s], ph)) { put_status(p.status, DEV_TIMEOUT_MMA); ok = false; break; }
            tc_fence_after();
            const uint64_t desc = umma_desc_k_sw128(smem_u32(smem + s * C::kStageBytes));
            if (leader) {
#pragma unroll
              for (int u = 0; u < KPS; ++u) {
                const uint64_t adesc = desc + u * (C::kSubBytes >> 4), bdesc = adesc + (kATileBytes >> 4);
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk) umma_bf16_pair(d, adesc + 2 * kk, bdesc + 2 * kk, idesc, ((kb - k0) | u | kk) != 0);
              }
              umma_commit_pair(&empty_bar[s]);
            }
            if (++s == STAGES) { s = 0; ph ^= 1; }
          }
          if (ok && leader) umma_commit_pair(&acc_full[buf]);
        }
    }
  } else {
    // ---- epilogue: thread = half of the tile's columns of one of this CTA's 128 rows ----
    pdl_wait();
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t lane_off = uint32_t(quarter * 32) << 16;
    uint32_t seg = 0;
    bool ok = true;
    for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
      const int m0 = (tile % tiles_m) * (2 * BM) + (int)rank * BM, n0 = (tile / tiles_m) * BN;
      const int row = m0 + quarter * 32 + lane, col0 = n0 + half * COLS;
      const bool row_ok = row < p.M;
      const int id = row_ok && p.ids ? dep_load(p.ids + row) : -1;
      float b[COLS / 32];                        // the bias of 32 columns in the warp's lanes
#pragma unroll
      for (int i = 0; i < COLS / 32; ++i) {
        const int col = col0 + lane + 32 * i;
        b[i] = col < p.N && p.bias ? load_bf16(p.bias + col) : 0.f;
      }
      float acc[COLS];
      for (int k0 = 0; k0 < num_kb; k0 += kSegmentBlocks, ++seg) {
        const uint32_t buf = seg & 1;
        if (ok && !mbar_wait(&acc_full[buf], (seg >> 1) & 1)) { put_status(p.status, DEV_TIMEOUT_EPI); ok = false; }
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t t0 = tmem_base + lane_off + buf * kAccStride + half * COLS;
        const bool first = k0 == 0;
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += 16) {
          uint32_t r[16];
          tmem_ld16(t0 + c0, r);
          tmem_wait_ld();
          if (c0 + 16 == COLS) { tc_fence_before(); mbar_arrive_cluster(&acc_empty[buf], 0); }
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c0 + i] = first ? __uint_as_float(r[i]) : acc[c0 + i] + __uint_as_float(r[i]);
        }
      }
      if (!ok) break;
      const int left = p.N - col0;               // columns of the row from here on
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        acc[i] += __shfl_sync(0xFFFFFFFFu, b[i / 32], i & 31);
        if (i >= left) acc[i] = -INFINITY;
        m = fmaxf(m, acc[i]);
      }
      if (row_ok) {
        const float m0 = safe_max(m);
        uint64_t s2[2] = {0, 0}, t2[2] = {0, 0};
        const auto sum = [&](auto ex) {
#pragma unroll
          for (int i = 0; i < COLS; i += 2) {
            const uint64_t d = ex(pack2(acc[i], acc[i + 1])), e = exp2_pair(d);
            float x, y;
            unpack2(d, x, y);
            s2[i / 2 & 1] = add2(s2[i / 2 & 1], e);
            t2[i / 2 & 1] = fma2(e, pack2(fmaxf(x, -1e30f), fmaxf(y, -1e30f)), t2[i / 2 & 1]);   // (columns behind the last: -inf)
          }
        };
        struct { uint64_t s[2], t[2]; } sums;
        float dl = 0.f;
        if (is_near(m0, p.c)) {
          const float R = reference(m0, p.c);
          sum(Expo<true>(R, p.c));
          dl = delta(m0, p.c, R);
        } else {
          sum(Expo<false>(m0, p.c));
        }
        sums.s[0] = s2[0]; sums.s[1] = s2[1]; sums.t[0] = t2[0]; sums.t[1] = t2[1];
        const Part part = part_of(m, sums, dl);
        p.part[(size_t)((tile / tiles_m) * 2 + half) * p.M + row] = make_float4(part.m, part.s, part.t, 0.f);
      }
      const int at = id - col0;
      if (at >= 0 && at < min(COLS, left)) p.xid[row] = pick<COLS>(acc, at);
    }
  }
  // Neither CTA may leave (or free tensor memory) while the other can still signal it or read its operands.
  tc_fence_before();
  cluster_sync_all();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

// The row's parts put together.  A CTA has R rows, neighbouring threads neighbouring rows; its 256 / R threads of a row take the parts in turn.  32 rows where there are
// few parts; 8 where there are 64 or more, of which a thread would else read a long chain.  us of both launches, 8 rows / 32, C 512: 1000 rows of 2048 (32 parts) 8.8 / 8.2, of 4096 (32) 12.3 / 11.4, of 8192 (64) 16.9 / 18.3, of 16384
// (128) 25.9 / 29.3; 300 rows of 2048 (32) 7.6 / 7.5, of 4096 (64) 8.3 / 8.6, of 16384 (128) 17.7 / 21.2, of 65536 (512) 42 / 58.
constexpr int kFinishThreads = 256, kFinishWarps = kFinishThreads / 32, kManyParts = 64;
struct FinishArgs {
  const float4* part; const float* xid; const int32_t* ids;
  int M, N, parts;
  float c, inv_tau;
  float* logprob; float2* stats; float* entropy;
  int32_t* status;
};
template <int R> __global__ void __launch_bounds__(kFinishThreads) linear_finish_kernel(const FinishArgs p) {
  constexpr int PER = kFinishThreads / R;          // threads of a row
  __shared__ Part all[kFinishWarps][R];
  pdl_trigger();
  const int warp = threadIdx.x >> 5, r = threadIdx.x % R, row = blockIdx.x * R + r;
  const bool row_ok = row < p.M;
  pdl_wait();
  const auto join = [&](const Part& a, const Part& b) {
    const float m = fmaxf(a.m, b.m);
    const Part x = against<true>(a, m, p.c), y = against<true>(b, m, p.c);
    return Part{m, x.s + y.s, x.t + y.t};
  };
  Part mine{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x / R; row_ok && i < p.parts; i += 4 * PER) {
    float4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * PER < p.parts) v[j] = dep_load4(p.part + (size_t)(i + j * PER) * p.M + row);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * PER < p.parts) mine = join(mine, Part{v[j].x, v[j].y, v[j].z});
  }
  __syncwarp();
#pragma unroll
  for (int o = 16; o >= R; o >>= 1)
    mine = join(mine, Part{__shfl_xor_sync(0xFFFFFFFFu, mine.m, o), __shfl_xor_sync(0xFFFFFFFFu, mine.s, o), __shfl_xor_sync(0xFFFFFFFFu, mine.t, o)});
  if ((threadIdx.x & 31) < R) all[warp][r] = mine;
  __syncthreads();
  if (threadIdx.x >= R || !row_ok) return;
#pragma unroll
  for (int w = 1; w < kFinishWarps; ++w) mine = join(mine, all[w][r]);
  const Stat st = stat_of<true>(mine.m, mine.s, mine.t);
  if (p.stats) p.stats[row] = make_float2(st.m, st.L);
  if (p.entropy) p.entropy[row] = st.H;
  if (!p.logprob) return;
  const int id = dep_load(p.ids + row);
  float lp = 0.f;
  if (id >= 0 && id < p.N) {
    lp = st.L == -INFINITY ? -INFINITY : (dep_load(p.xid + row) - st.m) * p.inv_tau - st.L;   // (a bias may forbid tokens)
  } else if (id != -1) {
    put_status(p.status, DEV_BAD_TOKEN_ID);
    lp = __int_as_float(0x7FC00000);
  }
  p.logprob[row] = lp;
}

// Tile width: the cheaper by rounds, one of 128 columns costing 0.62 of one of 256 (us, 256 / 128 wide: 400 rows, C 2048, V 4096 17.6 / 12.8; 820 18.6 / 20.6; 5000, C 256,
// V 1000 15.0 / 12.9; 8192, C 2048, V 4096 95 / 115; tiles of 64 columns were never faster).
int tile_width(int M, int N) {
  const auto rounds = [&](int bn) { return (((long)(M + 2 * BM - 1) / (2 * BM)) * ((N + bn - 1) / bn) + 73) / 74; };
  return 0.62 * rounds(128) < rounds(256) ? 128 : 256;
}
int column_parts(int M, int N) { const int bn = tile_width(M, N); return 2 * ((N + bn - 1) / bn); }

template <int BN> cudaError_t allow_smem() { return cudaFuncSetAttribute(linear_logprobs_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<BN>::kSmem); }
// Function attributes belong to a device: set on the first call on each.
cudaError_t linear_init() {
  static std::atomic<uint64_t> done{0};
  return once_per_device(done, [] {
    const cudaError_t e = allow_smem<256>();
    return e == cudaSuccess ? allow_smem<128>() : e;
  });
}

template <int BN> cudaError_t launch_width(const void* a, const void* w, const LinearArgs& p, cudaStream_t st) {
  alignas(64) CUtensorMap tmA, tmB;
  if (!make_tmap_bf16_2d(&tmA, a, p.M, p.K, BM) || !make_tmap_bf16_2d(&tmB, w, p.N, p.K, BN / 2)) return cudaErrorInvalidValue;
  const long tiles = (long)((p.M + 2 * BM - 1) / (2 * BM)) * ((p.N + BN - 1) / BN);
  const int pairs = (int)(tiles < 74 ? tiles : 74);
  return launch_pdl(linear_logprobs_kernel<BN>, dim3(2 * pairs), dim3(kThreads), Cfg<BN>::kSmem, st, tmA, tmB, p);
}

// Few rows: the product with K split over a cluster (fv_gemm_bf16; its slices are at most 512 of K for these sizes, so its sums are as exact) and the rows read back from
// L2, which is sooner done than 256-row tiles while weights bound both.  us, this route / tiles, 1, 16, 32, 48 rows: C 1024, V 4096 5.6 / 10.9, 6.3 / 9.4, 6.4 / 9.4, 7.7 / 9.5; C 2048, V 4096 7.7 / 18.1,
// 8.2 / 13.8, 8.2 / 13.4, 9.6 / 13.3; C 2048, V 9472 14.7 / 23.1, 15.2 / 18.8, 15.2 / 15.7, 17.7 / 16.0; C 512, V 9472 9.5 / 10.0, 10.3 / 9.9, 10.8 / 10.3, 12.7 / 10.6: 48 rows of many columns are where it loses.
// Beyond these limits fv_gemm_bf16 adds more of K in one piece, so that such calls take the tiles although it would be sooner done for some (128 rows, C 2048, V 4096 11.9 / 13.5; one row, C 1024, V 16384 9.5 / 17.2,
// V 65536 33 / 50; one row, C 4096, V 4096 10.5 / 27.3), with up to five times the error of their logits.
constexpr int kFewRows = 48, kFewColumns = 9472, kFewK = 2048;
size_t few_rows_bytes(int rows, int V) { return rows <= kFewRows && V <= kFewColumns ? (size_t)rows * V * 4 : 0; }

// Rows, channels, columns and tiles are counted in 32 bits, a tile or a block of K past the last.
constexpr int kMostSize = INT_MAX - 255;
bool too_large(int rows, int V) { return rows > kMostSize || V > kMostSize || (long long)((rows + 255) / 256) * ((V + 127) / 128) > kMostSize; }

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace fv

using namespace fv;

extern "C" {

size_t fv_linear_logprobs_workspace_bytes(int32_t rows, int32_t V) {
  if (rows <= 0 || V <= 0 || too_large(rows, V)) return 0;
  const size_t parts = align_up((size_t)rows * column_parts(rows, V) * sizeof(float4), 256) + align_up((size_t)rows * 4, 256);
  return std::max(parts, align_up(few_rows_bytes(rows, V), 256));
}

fv_status fv_linear_logprobs(const void* a_dev, const void* w_dev, const void* bias_dev, int32_t rows, int32_t C, int32_t V, float tau, const int32_t* ids_dev,
                             float* logprob_out_dev, float* stats_out_dev, float* entropy_out_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                             void* stream) {
  if (!a_dev || !w_dev || rows <= 0 || C <= 0 || (C % 8) || V <= 0 || (V % 8) || !(tau >= 1e-6f && tau <= 1e6f)) return FV_ERR_INVALID_ARG;
  if (!aligned_to(a_dev, 16) || !aligned_to(w_dev, 16) || !aligned_to(bias_dev, 16) || !workspace_dev || !aligned_to(workspace_dev, 256)) return FV_ERR_INVALID_ARG;
  if ((ids_dev != nullptr) != (logprob_out_dev != nullptr) || !aligned_to(stats_out_dev, 8) || (!logprob_out_dev && !stats_out_dev && !entropy_out_dev)) return FV_ERR_INVALID_ARG;
  if (C > kMostSize || too_large(rows, V)) return FV_ERR_UNSUPPORTED;
  if (workspace_bytes < fv_linear_logprobs_workspace_bytes(rows, V)) return FV_ERR_CAPACITY;
  if (C <= kFewK && few_rows_bytes(rows, V) > 0) {
    const fv_status s = fv_gemm_bf16(a_dev, w_dev, bias_dev, rows, V, C, EPI_F32, workspace_dev, nullptr, nullptr, 0, rows, status_dev, nullptr, 0, stream);
    if (s != FV_OK) return s;
    return fv_token_logprobs(workspace_dev, 0, V, rows, V, tau, ids_dev, 0, logprob_out_dev, stats_out_dev, entropy_out_dev, nullptr, nullptr, status_dev, stream);
  }
  if (linear_init() != cudaSuccess) return FV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  float4* part = static_cast<float4*>(workspace_dev);
  float* xid = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + align_up((size_t)rows * column_parts(rows, V) * sizeof(float4), 256));
  const int bn = tile_width(rows, V), parts = column_parts(rows, V);
  {
    LaunchScope scope(KC_GEMM, 1, 2.0 * rows * (double)V * C, 2.0 * ((double)rows * C + (double)V * C) + 16.0 * rows * parts, st);
    const LinearArgs p{rows, V, C, kLog2e * (1.f / tau), static_cast<const __nv_bfloat16*>(bias_dev), ids_dev, part, xid, status_dev};
    const cudaError_t e = bn == 256 ? launch_width<256>(a_dev, w_dev, p, st) : launch_width<128>(a_dev, w_dev, p, st);
    if (e != cudaSuccess) return FV_ERR_CUDA;
  }
  const double bytes = 16.0 * rows * parts + 20.0 * rows;
  LaunchScope scope(KC_SELECT, 1, bytes, bytes, st);
  const FinishArgs f{part, xid, ids_dev, rows, V, parts, kLog2e * (1.f / tau), 1.f / tau, logprob_out_dev, reinterpret_cast<float2*>(stats_out_dev), entropy_out_dev, status_dev};
  const cudaError_t e = parts < kManyParts ? launch_pdl(linear_finish_kernel<32>, dim3((unsigned)((rows + 31) / 32)), dim3(kFinishThreads), 0, st, f)
                                           : launch_pdl(linear_finish_kernel<8>, dim3((unsigned)((rows + 7) / 8)), dim3(kFinishThreads), 0, st, f);
  return e == cudaSuccess ? FV_OK : FV_ERR_CUDA;
}

}  // extern "C"
