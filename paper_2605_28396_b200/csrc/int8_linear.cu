// Products in 8-bit integers: rows quantised with a step each, and out = (x w^T) in whole numbers times the
// two rows' steps.  It is the output projection of a frozen policy whose embedding is kept in 8 bits.
//
// quantize_rows_kernel:  step = max|x| / 127,  q = x / step to the nearest whole number, ties to even, within
// [-127, 127], both divisions correctly rounded in fp32, so that every implementation of this definition gets the same q.
//
// linear_i8_few_kernel (up to 16 rows of x): one pass over w, memory-bound; see there.
//
// linear_i8_kernel: tcgen05.mma kind::i8 on CTA pairs, 256 x 256 tiles, accumulators of 32-bit whole numbers
// in tensor memory (exact: d < 2^17 keeps every sum below 2^31), operands by TMA in the 128-byte
// swizzle, 128 entries of the contraction a k-block.  The pipeline is that of tc_pipeline.cuh: bytes
// are laid out as for 64 bf16.  An accumulator becomes float(acc) * (step_x * step_w): three roundings.
// The results leave through shared memory as whole pieces of rows: 4 096 x 2 560 against 151 936 channels 1.11 to 1.18 ms in a
// captured graph on a cool GPU (2.7 to 2.9 POP/s), 1.22 to 1.27 in a series of calls at the power limit, where 16-byte stores of
// a lane's own row took 1.19 to 1.23; 777 x 1 000 against 50 257 channels (rows off 16-byte boundaries, fp32) 81 to 88 us,
// 294 with scattered 4-byte stores, 114 in pieces of 32.
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

// (a subnormal step is rounded by up to half a unit of 2^-149: the largest entry may be more than 127 of it)
__device__ __forceinline__ int quantized(float x, float step) {
  return max(-127, min(127, __float2int_rn(__fdiv_rn(x, step))));
}

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
  bool whole;          // rows of out start on 16-byte boundaries
  int32_t* status;
  uint64_t limit_ns;
};
// Behind the stages: per epilogue warp 32 rows of 64 results on their way out (16-byte units XOR-swizzled with
// the row).
constexpr int kStages = 5;
template <typename TOut>
__host__ __device__ constexpr int out_row() { return 64 * (int)sizeof(TOut); }   // bytes: 64 results
constexpr int kWarpBytes = 32 * out_row<float>();
constexpr int kLinearSmem = kCtrlBytes + 1024 + kStages * kPairStageBytes + (kEpiThreads / 32) * kWarpBytes;
static_assert(kLinearSmem <= 227 * 1024 && kStages <= kPairStages, "shared memory");

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
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!bar_wait(smem_addr(&ctrl->empty[s]), ph ^ 1, abort, p.limit_ns)) { ok = false; break; }
          const uint32_t bar = smem_addr(&ctrl->full[s]);
          const uint32_t a = stage0 + s * kPairStageBytes, b = a + kABytes;
          if (rank == 0) bar_expect_tx(bar, 2 * kPairStageBytes);
          const uint32_t bar0 = map_to_cta(bar, 0);
          tma_load_2d_pair(a, &map_x, kb * kBKBytes, m0, bar0);
          tma_load_2d_pair(b, &map_w, kb * kBKBytes, n0, bar0);
        }
      }
      pair_issued(ctrl, rank, it);
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
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
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
    }
  } else if (warp >= kEpiWarp0) {
    // A lane holds a row of the accumulator.  Its results go through shared memory, so that they leave
    // as whole pieces of rows: 16 bytes a lane along a row where rows start on 16-byte boundaries, an
    // entry a lane otherwise.
    const int quad = warp & 3, half = (warp - kEpiWarp0) >> 2;
    uint8_t* const mine = smem_raw + (stage0 - smem_addr(smem_raw)) + kStages * kPairStageBytes + (warp - kEpiWarp0) * kWarpBytes;
    constexpr int kOutRow = out_row<TOut>(), kUnits = kOutRow / 16, kPass = 64;   // columns that go out at a time
    uint32_t acc_it = 0;
    for (int64_t t = pair; t < tiles; t += pairs, ++acc_it) {
      int pm, nt;
      tile_of(p, t, pm, nt);
      const uint32_t slot = acc_it & 1, aph = (acc_it >> 1) & 1;
      const int64_t m0 = (int64_t)(2 * pm + (int)rank) * kBM + quad * 32, n0 = (int64_t)nt * kBN + half * 128;
      const int rows = p.M - m0 < 32 ? (p.M > m0 ? (int)(p.M - m0) : 0) : 32;
      const int cols = p.N - n0 < 128 ? (p.N > n0 ? (int)(p.N - n0) : 0) : 128;
      // (the steps are asked for while the tile is on its way)
      const float sx = lane < rows ? __ldg(p.step_x + m0 + lane) : 0.f;
      float steps[4];   // of columns lane, 32 + lane, ...
#pragma unroll
      for (int j = 0; j < 4; ++j) steps[j] = j * 32 + lane < cols ? __ldg(p.step_w + n0 + j * 32 + lane) : 0.f;
      if (!__all_sync(0xffffffffu, bar_wait(smem_addr(&ctrl->acc_full[slot]), aph, abort, p.limit_ns))) break;
      tc_fence_after_sync();
      const uint32_t t_lane = tmem_base + ((uint32_t)(quad * 32) << 16) + slot * kBN + (uint32_t)(half * 128);
      const int passes = rows > 0 ? (cols + kPass - 1) / kPass : 0;
#pragma unroll 1
      for (int pass = 0; pass < passes; ++pass) {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kPass / 32; ++j) {
          uint32_t r[32];
          tmem_ld32(t_lane + pass * kPass + j * 32, r);
          tmem_ld_wait();
          const float sw = pass == 0 ? steps[j] : steps[2 + j];
          constexpr int kUnit = 16 / (int)sizeof(TOut);   // results of a 16-byte unit
#pragma unroll
          for (int u = 0; u < 32 / kUnit; ++u) {
            float v[kUnit];
#pragma unroll
            for (int i = 0; i < kUnit; ++i)
              v[i] = (float)(int)r[u * kUnit + i] * (sx * __shfl_sync(0xffffffffu, sw, u * kUnit + i));
            uint4 x;
            if (sizeof(TOut) == 2)
              x = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4 % kUnit], v[5 % kUnit]),
                             pack_bf16x2(v[6 % kUnit], v[7 % kUnit]));
            else
              x = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            const int unit = j * (32 / kUnit) + u;
            *reinterpret_cast<uint4*>(mine + lane * kOutRow + ((unit ^ (lane & (kUnits - 1))) << 4)) = x;
          }
        }
        __syncwarp();
        const int left = cols - pass * kPass < kPass ? cols - pass * kPass : kPass;
        TOut* o = static_cast<TOut*>(p.out) + m0 * p.ldo + n0 + pass * kPass;
        if (p.whole && left == kPass) {
          const int unit = lane % kUnits;
          for (int i = lane / kUnits; i < rows; i += 32 / kUnits) {
            const uint4 x = *reinterpret_cast<const uint4*>(mine + i * kOutRow + ((unit ^ (i & (kUnits - 1))) << 4));
            __stcs(reinterpret_cast<uint4*>(o + i * p.ldo) + unit, x);
          }
        } else {
          for (int i = 0; i < rows; ++i) {
            const TOut* row = reinterpret_cast<const TOut*>(mine + i * kOutRow);
            constexpr int kUnit = 16 / (int)sizeof(TOut);
#pragma unroll
            for (int k = 0; k < kPass / 32; ++k) {
              const int c = k * 32 + lane;
              if (c < left) o[i * p.ldo + c] = row[((c / kUnit) ^ (i & (kUnits - 1))) * kUnit + c % kUnit];
            }
          }
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) pair_release(&ctrl->acc_empty[slot], rank);
    }
  }
  pair_finish<kStages>(ctrl, rank, p.status);
}

// ---------------------------------------------------------------------------- few rows of x
// Up to 16 tokens (decoding): W passes through once and bounds the call, and tensor-memory tiles would be
// nearly empty.  Four warps take 16 rows of W, a quarter of the contraction each, straight from global memory into
// the operand registers of mma.sync (any order of the contraction will do, as long as both operands have it:
// a thread's 16 bytes of a row are its share of two instructions); x lies in shared memory.
constexpr int kFewThreads = 512, kFewCtas = 2;
constexpr int kFewGroups = kFewThreads / 128;
constexpr int kFewMax = 16;          // tokens
constexpr int kFewUnroll = 5;        // 64-byte blocks of a row in flight per warp, two loads each
constexpr int kFewSmemX = 96 * 1024;

struct FewParams {
  const int8_t *x, *w;
  int64_t ldx, ldw, N;
  int M, d, pitch;     // pitch: bytes from row to row of x in shared memory, 64 more than a multiple of 128
  const float *step_x, *step_w;
  void* out;
  int64_t ldo;
  int32_t* status;
};

__device__ __forceinline__ void mma_i8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename TOut, int NT>   // NT: 8-token tiles
__global__ void __launch_bounds__(kFewThreads, kFewCtas) linear_i8_few_kernel(const FewParams p) {
  chain();
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* xs = smem_raw;
  int* part = reinterpret_cast<int*>(smem_raw + NT * 8 * p.pitch);   // [group][parity][3][NT * 4][32]
  const int tid = threadIdx.x, lane = tid & 31, group = tid >> 7, quarter = (tid >> 5) & 3;
  const int pieces = p.pitch / 16;
  for (int i = tid; i < NT * 8 * pieces; i += kFewThreads) {
    const int row = i / pieces, k = (i % pieces) * 16;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (row < p.M && k < p.d) {
      v = __ldg(reinterpret_cast<const uint4*>(p.x + (int64_t)row * p.ldx + k));
      const int n = p.d - k;          // bytes behind the row's d count as zeros
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n < 4 * j + 4) w[j] = n <= 4 * j ? 0u : w[j] & ((1u << (8 * (n - 4 * j))) - 1u);
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *reinterpret_cast<uint4*>(xs + row * p.pitch + k) = v;
  }
  __syncthreads();
  const int g = lane >> 2, t = lane & 3;
  const int d16 = (p.d + 15) & ~15, blocks = (p.d + 63) / 64;
  const uint8_t* xl = xs + g * p.pitch + t * 16;
  const int64_t tiles = (p.N + 15) / 16, step = (int64_t)gridDim.x * kFewGroups;
  int par = 0;
  for (int64_t tile = (int64_t)blockIdx.x * kFewGroups + group; tile < tiles; tile += step, par ^= 1) {
    const int64_t n0 = tile * 16 + g, n1 = n0 + 8;
    const int8_t* w0 = p.w + (n0 < p.N ? n0 : p.N - 1) * p.ldw + t * 16;
    const int8_t* w1 = p.w + (n1 < p.N ? n1 : p.N - 1) * p.ldw + t * 16;
    int acc[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = 0;
#pragma unroll 1
    for (int kb = quarter; kb < blocks; kb += 4 * kFewUnroll) {
      uint4 a[kFewUnroll], b[kFewUnroll];
#pragma unroll
      for (int u = 0; u < kFewUnroll; ++u) {
        const int k = (kb + 4 * u) * 64;
        a[u] = b[u] = make_uint4(0u, 0u, 0u, 0u);
        if (k + t * 16 < d16) {       // (a row's last bytes up to a multiple of 16 are there: its stride is one)
          a[u] = __ldcs(reinterpret_cast<const uint4*>(w0 + k));
          b[u] = __ldcs(reinterpret_cast<const uint4*>(w1 + k));
        }
      }
#pragma unroll
      for (int u = 0; u < kFewUnroll; ++u) {
        const int k = (kb + 4 * u) * 64;
        if (k >= p.d) break;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint4 x = *reinterpret_cast<const uint4*>(xl + i * 8 * p.pitch + k);
          mma_i8(acc[i], a[u].x, b[u].x, a[u].y, b[u].y, x.x, x.y);
          mma_i8(acc[i], a[u].z, b[u].z, a[u].w, b[u].w, x.z, x.w);
        }
      }
    }
    int* mine = part + ((group * 2 + par) * 3) * (NT * 4 * 32) + lane;
    if (quarter != 0) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mine[((quarter - 1) * NT * 4 + i * 4 + j) * 32] = acc[i][j];
    }
    asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory");
    if (quarter == 0) {   // (the others go on; this buffer is written again after the next meeting)
      const float s0 = n0 < p.N ? __ldg(p.step_w + n0) : 0.f, s1 = n1 < p.N ? __ldg(p.step_w + n1) : 0.f;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          int v = acc[i][j];
#pragma unroll
          for (int q = 0; q < 3; ++q) v += mine[(q * NT * 4 + i * 4 + j) * 32];
          const int m = i * 8 + t * 2 + (j & 1);
          const int64_t n = j < 2 ? n0 : n1;
          if (m < p.M && n < p.N)
            Elem<TOut>::store1(p.out, m * p.ldo + n, (float)v * (__ldg(p.step_x + m) * (j < 2 ? s0 : s1)));
        }
      }
    }
  }
}

template <typename TOut, int NT>
cudaError_t launch_few(const FewParams& p, int sm_count, cudaStream_t s) {
  const size_t smem = (size_t)NT * 8 * p.pitch + (size_t)kFewGroups * 2 * 3 * NT * 4 * 32 * 4;
  constexpr size_t limit = kFewSmemX + (size_t)kFewGroups * 2 * 3 * NT * 4 * 32 * 4;
  const cudaError_t e = shared_limit<linear_i8_few_kernel<TOut, NT>>(limit);
  if (e != cudaSuccess) return e;
  int64_t grid = (int64_t)sm_count * kFewCtas, tiles = ((p.N + 15) / 16 + kFewGroups - 1) / kFewGroups;
  if (grid > tiles) grid = tiles;
  return launch_chained(linear_i8_few_kernel<TOut, NT>, (unsigned)grid, kFewThreads, smem, 1, s, p);
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
  // few tokens, d = 2 560 against 151 936 channels (389 MB: 59 us at the copy rate): 8 take 100 us on the tiles,
  // 66 here, 16 98 and 75, 32 92 and 155; on the tiles 64 take 90, 128 97 and 256 107 (their rounding to 8 bits included)
  const int64_t row64 = (d + 63) / 64 * 64, pitch = row64 % 128 ? row64 : row64 + 64;
  const int tiles8 = (int)((M + 7) / 8);
  if (M <= kFewMax && tiles8 * 8 * pitch <= kFewSmemX) {
    const FewParams f = {x, w, ldx, ldw, N, (int)M, (int)d, (int)pitch, step_x, step_w, out, ldo, status};
    const bool bf = out_dtype == ADWIN_BF16;
    if (tiles8 == 1) return bf ? launch_few<__nv_bfloat16, 1>(f, sm_count, s) : launch_few<float, 1>(f, sm_count, s);
    return bf ? launch_few<__nv_bfloat16, 2>(f, sm_count, s) : launch_few<float, 2>(f, sm_count, s);
  }
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
  p.whole = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && (ldo * (out_dtype == ADWIN_BF16 ? 2 : 4)) % 16 == 0;
  p.status = status;
  p.limit_ns = handshake_wait_limit_ns();
  CUtensorMap mx, mw;
  if (!make_map_i8(&mx, x, d, M, ldx, kBM) || !make_map_i8(&mw, w, d, N, ldw, kBM)) return cudaErrorInvalidValue;
  const bool bf = out_dtype == ADWIN_BF16;
  const cudaError_t e = bf ? shared_limit<linear_i8_kernel<__nv_bfloat16>>(kLinearSmem)
                           : shared_limit<linear_i8_kernel<float>>(kLinearSmem);
  if (e != cudaSuccess) return e;
  return launch_chained(bf ? linear_i8_kernel<__nv_bfloat16> : linear_i8_kernel<float>, (unsigned)(sm_count & ~1),
                        kThreads, kLinearSmem, 2, s, mx, mw, p);
}

}  // namespace adwin
