// Products in 8-bit integers: rows quantised with a step each, and out = (x w^T) in whole numbers times the
// two rows' steps.  It is the output projection of a frozen policy whose embedding is kept in 8 bits.
//
// quantize_rows_kernel:  step = max|x| / 127,  q = x / step to the nearest whole number, ties to even,
// both divisions correctly rounded in fp32, so that every implementation of this definition gets the same q.
//
// linear_i8_kernel: tcgen05.mma kind::i8 on CTA pairs, 256 x 256 tiles, accumulators of 32-bit whole numbers
// in tensor memory (exact: d < 2^17 keeps every sum below 2^31), operands by TMA in the 128-byte
// swizzle, 128 entries of the contraction a k-block.  The pipeline is that of tc_pipeline.cuh: bytes
// are laid out as for 64 bf16.  An accumulator becomes float(acc) * (step_x * step_w): three roundings.
#include <cuda_bf16.h>

#include "adwin_common.cuh"
#include "adwin_internal.h"
#include "exp_sums.cuh"
#include "tc_pipeline.cuh"

namespace adwin {

using namespace tc;

namespace {

// ---------------------------------------------------------------------------- rows to 8 bits
constexpr int kQuantThreads = 128;

struct QuantParams {
  const void* x;
  int64_t M, d, ldx;
  int8_t* q;
  int64_t ldq;
  float* step;
  int32_t* status;
};

__device__ __forceinline__ int quantized(float x, float step) { return __float2int_rn(__fdiv_rn(x, step)); }

template <typename TIn>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const QuantParams p) {
  chain();
  constexpr int N = Elem<TIn>::N;
  __shared__ float red[kQuantThreads / 32];
  const int tid = threadIdx.x;
  for (int64_t r = blockIdx.x; r < p.M; r += gridDim.x) {
    const char* row = static_cast<const char*>(p.x) + (size_t)r * p.ldx * sizeof(TIn);
    int8_t* out = p.q + (size_t)r * p.ldq;
    const bool vec = (reinterpret_cast<uintptr_t>(row) & 15) == 0 && (reinterpret_cast<uintptr_t>(out) & (N - 1)) == 0;
    const int64_t pieces = vec ? p.d / N : 0;
    float m = 0.f;
    for (int64_t i = tid; i < pieces; i += kQuantThreads) {
      float x[N];
      Elem<TIn>::unpack(__ldg(reinterpret_cast<const uint4*>(row) + i), x);
#pragma unroll
      for (int j = 0; j < N; ++j) m = max_nan(m, fabsf(x[j]));
    }
    for (int64_t i = pieces * N + tid; i < p.d; i += kQuantThreads) m = max_nan(m, fabsf(Elem<TIn>::load1(row, i)));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((tid & 31) == 0) red[tid >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / 32; ++w) m = max_nan(m, red[w]);
    const bool finite = isfinite(m);
    const float step = finite ? __fdiv_rn(m, 127.f) : __int_as_float(0x7fc00000);
    const bool some = step > 0.f;   // (a row of zeros, or too small for a step, or not finite: all 0)
    for (int64_t i = tid; i < pieces; i += kQuantThreads) {
      float x[N];
      Elem<TIn>::unpack(__ldg(reinterpret_cast<const uint4*>(row) + i), x);
      uint32_t w[N / 4];
#pragma unroll
      for (int j = 0; j < N / 4; ++j) {
        w[j] = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[j] |= ((uint32_t)(some ? quantized(x[4 * j + k], step) : 0) & 0xffu) << (8 * k);
      }
      if (N == 8) reinterpret_cast<uint2*>(out)[i] = make_uint2(w[0], w[N / 4 - 1]);
      else reinterpret_cast<uint32_t*>(out)[i] = w[0];
    }
    for (int64_t i = pieces * N + tid; i < p.d; i += kQuantThreads)
      out[i] = (int8_t)(some ? quantized(Elem<TIn>::load1(row, i), step) : 0);
    if (tid == 0) {
      p.step[r] = step;
      if (!finite) atomicOr(p.status, (int32_t)ADWIN_DEV_NONFINITE);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------- product
constexpr int kBKBytes = 128;        // entries of the contraction of a k-block
constexpr int kGroupM = 16;          // 256-row tiles that share their passes over W

// Instruction descriptor of tcgen05.mma.kind::i8, M = 256, N = 256: accumulator of 32-bit whole numbers
// (bits 4..5 = 2), A and B signed 8-bit (bits 7..9, 10..12 = 1), both K-major, N >> 3, M >> 4.
constexpr uint32_t kDescI8 =
    (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kBN >> 3) << 17) | ((uint32_t)(2 * kBM >> 4) << 24);

__device__ __forceinline__ void umma_i8_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(kDescI8), "r"(accumulate)
      : "memory");
}

struct LinearParams {
  int64_t M, N;
  int m_pairs, n_tiles, k_blocks;
  const float *step_x, *step_w;
  void* out;
  int64_t ldo;
  int32_t* status;
  uint64_t limit_ns;
};

// Tile t: groups of kGroupM row tiles, within one the row tiles of a column tile follow one another, so
// that W passes through once a group and the group's rows of x stay in L2.
__device__ __forceinline__ void tile_of(const LinearParams& p, int64_t t, int& pm, int& n) {
  const int64_t per = (int64_t)kGroupM * p.n_tiles;
  const int g = (int)(t / per);
  const int64_t u = t - g * per;
  const int rows = p.m_pairs - g * kGroupM < kGroupM ? p.m_pairs - g * kGroupM : kGroupM;
  pm = g * kGroupM + (int)(u % rows);
  n = (int)(u / rows);
}

template <typename TOut>
__global__ void __launch_bounds__(kThreads, 1)
linear_i8_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                 const LinearParams p) {
  chain_wait();
  extern __shared__ uint8_t smem_raw[];
  Ctrl* ctrl = reinterpret_cast<Ctrl*>(smem_raw);
  const uint32_t stage0 = (smem_addr(smem_raw) + kCtrlBytes + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &ctrl->abort;
  const uint32_t rank = cluster_ctarank();

  if (threadIdx.x == 0) pair_bars_init(ctrl);
  if (warp == 2) {
    tmem_alloc_pair(smem_addr(&ctrl->tmem_base), kTmemCols);
    tmem_relinquish_pair();
    tc_fence_before_sync();
  }
  __syncthreads();
  cluster_sync();
  tc_fence_after_sync();
  const uint32_t tmem_base = ctrl->tmem_base;
  const int64_t tiles = (int64_t)p.m_pairs * p.n_tiles;
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int64_t t = pair; ok && t < tiles; t += pairs) {
        int pm, n;
        tile_of(p, t, pm, n);
        const int m0 = (2 * pm + (int)rank) * kBM, n0 = n * kBN + (int)rank * (kBN / 2);
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % kPairStages, ph = (it / kPairStages) & 1;
          if (!bar_wait(smem_addr(&ctrl->empty[s]), ph ^ 1, abort, p.limit_ns)) { ok = false; break; }
          const uint32_t bar = smem_addr(&ctrl->full[s]);
          const uint32_t a = stage0 + s * kPairStageBytes, b = a + kABytes;
          if (rank == 0) bar_expect_tx(bar, 2 * kPairStageBytes);
          const uint32_t bar0 = map_to_cta(bar, 0);
          tma_load_2d_pair(a, &map_x, kb * kBKBytes, m0, bar0);
          tma_load_2d_pair(b, &map_w, kb * kBKBytes, n0, bar0);
        }
      }
      if (!ok && rank == 0) pair_drain_loads(ctrl, it);
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, acc_it = 0;
      bool ok = true;
      for (int64_t t = pair; ok && t < tiles; t += pairs, ++acc_it) {
        const uint32_t slot = acc_it & 1, aph = (acc_it >> 1) & 1;
        if (!bar_wait(smem_addr(&ctrl->acc_empty[slot]), aph ^ 1, abort, p.limit_ns)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t tmem_d = tmem_base + slot * kBN;
        for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
          const uint32_t s = it % kPairStages, ph = (it / kPairStages) & 1;
          if (!bar_wait(smem_addr(&ctrl->full[s]), ph, abort, p.limit_ns)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t a = stage0 + s * kPairStageBytes, b = a + kABytes;
          const uint64_t ad = desc_k_major(a), bd = desc_k_major(b);
#pragma unroll
          for (int k = 0; k < kBKBytes / 32; ++k)   // 32 bytes of the contraction an instruction
            umma_i8_pair(tmem_d, ad + (uint64_t)(k * kStepKMajor), bd + (uint64_t)(k * kStepKMajor),
                         (kb == 0 && k == 0) ? 0u : 1u);
          umma_commit_pair(smem_addr(&ctrl->empty[s]));
        }
        if (ok) umma_commit_pair(smem_addr(&ctrl->acc_full[slot]));
      }
      if (!ok) {
        umma_commit_pair(smem_addr(&ctrl->drain));
        bar_wait_drain(smem_addr(&ctrl->drain), 0);
      }
    }
  } else if (warp >= kEpiWarp0) {
    const int quad = warp & 3, half = (warp - kEpiWarp0) >> 2;
    const int row = quad * 32 + lane;
    uint32_t acc_it = 0;
    for (int64_t t = pair; t < tiles; t += pairs, ++acc_it) {
      int pm, nt;
      tile_of(p, t, pm, nt);
      const uint32_t slot = acc_it & 1, aph = (acc_it >> 1) & 1;
      const int64_t m = (int64_t)(2 * pm + (int)rank) * kBM + row;
      const int64_t n0 = (int64_t)nt * kBN + half * 128;
      const float sx = m < p.M ? p.step_x[m] : 0.f;
      TOut* o = static_cast<TOut*>(p.out) + (m < p.M ? m : 0) * p.ldo + n0;
      const bool wide = (reinterpret_cast<uintptr_t>(o) & 15) == 0;
      if (!__all_sync(0xffffffffu, bar_wait(smem_addr(&ctrl->acc_full[slot]), aph, abort, p.limit_ns))) break;
      tc_fence_after_sync();
      const uint32_t t_lane = tmem_base + ((uint32_t)(quad * 32) << 16) + slot * kBN + (uint32_t)(half * 128);
#pragma unroll 1
      for (int j = 0; j < 4; ++j) {
        uint32_t r[32];
        __syncwarp();   // (lanes without a row come back here: the load is the warp's)
        tmem_ld32(t_lane + j * 32, r);
        tmem_ld_wait();
        const int64_t nj = n0 + j * 32;
        const int left = nj >= p.N ? 0 : (p.N - nj < 32 ? (int)(p.N - nj) : 32);
        if (m >= p.M || left == 0) continue;
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i)
          v[i] = (float)(int)r[i] * (sx * (i < left ? __ldg(p.step_w + nj + i) : 0.f));
        TOut* oj = o + j * 32;
        if (wide && left == 32) {
          if (sizeof(TOut) == 2) {
#pragma unroll
            for (int i = 0; i < 32; i += 8)
              *reinterpret_cast<uint4*>(oj + i) =
                  make_uint4(pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]),
                             pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7]));
          } else {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<float4*>(oj + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < left) Elem<TOut>::store1(oj, i, v[i]);
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) pair_release(&ctrl->acc_empty[slot], rank);
    }
  }
  if (*abort && threadIdx.x == 0) {
    atomicOr(p.status, ADWIN_DEV_TIMEOUT);
    store_cluster_u32(map_to_cta(smem_addr(&ctrl->abort), rank ^ 1u), 1u);
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();
  if (warp == 2) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

}  // namespace

cudaError_t launch_quantize_rows(const void* x, int dtype, int64_t M, int64_t d, int64_t ldx, int8_t* q,
                                 int64_t ldq, float* step, int32_t* status, int sm_count, cudaStream_t s) {
  const QuantParams p = {x, M, d, ldx, q, ldq, step, status};
  int64_t grid = (int64_t)sm_count * 64;
  if (grid > M) grid = M;
  return dtype == ADWIN_BF16
             ? launch_chained(quantize_rows_kernel<__nv_bfloat16>, (unsigned)grid, kQuantThreads, 0, 1, s, p)
             : launch_chained(quantize_rows_kernel<float>, (unsigned)grid, kQuantThreads, 0, 1, s, p);
}

cudaError_t launch_linear_i8(const int8_t* x, int64_t ldx, const float* step_x, const int8_t* w, int64_t ldw,
                             const float* step_w, int64_t M, int64_t N, int64_t d, void* out, int out_dtype,
                             int64_t ldo, int32_t* status, int sm_count, cudaStream_t s) {
  LinearParams p = {};
  p.M = M;
  p.N = N;
  p.m_pairs = (int)((M + 2 * kBM - 1) / (2 * kBM));
  p.n_tiles = (int)((N + kBN - 1) / kBN);
  p.k_blocks = (int)((d + kBKBytes - 1) / kBKBytes);
  p.step_x = step_x;
  p.step_w = step_w;
  p.out = out;
  p.ldo = ldo;
  p.status = status;
  p.limit_ns = handshake_wait_limit_ns();
  CUtensorMap mx, mw;
  if (!make_map_i8(&mx, x, d, M, ldx, kBM) || !make_map_i8(&mw, w, d, N, ldw, kBM)) return cudaErrorInvalidValue;
  return out_dtype == ADWIN_BF16 ? launch_pairs(linear_i8_kernel<__nv_bfloat16>, sm_count, s, mx, mw, p)
                                 : launch_pairs(linear_i8_kernel<float>, sm_count, s, mx, mw, p);
}

}  // namespace adwin
