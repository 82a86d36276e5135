// The rows a call works on, found by every CTA for itself: the operators that read a teacher's or a
// policy's scores take no workspace, so there is no row map in memory to look a row up in.
//
// Up to kListMax sequences a CTA forms the prefix sums of the processed ranges in shared memory
// (one load per sequence, a scan by one warp) and walks the compact list, which keeps the rows of
// ragged windows evenly spread.  With more sequences, or none that is cut short, it walks all
// positions and skips those outside.
#pragma once

#include "adwin_common.cuh"

namespace adwin {

constexpr int kListMax = 256;

struct RowRange {
  const int32_t* window;    // [B] or null (= T)
  const int32_t* rollout;   // [B] or null (= T)
  int64_t B, T;
  // End of sequence b's processed range; *bad is set where a length is invalid (it is clamped).
  __device__ __forceinline__ int64_t end(int64_t b, bool& bad) const {
    int64_t W = window ? (int64_t)window[b] : T, R = rollout ? (int64_t)rollout[b] : T;
    bad = W < 0 || R < 0 || R > T;
    R = R < 0 ? 0 : (R > T ? T : R);
    W = W < 0 ? 0 : W;
    return W < R ? W : R;
  }
  __device__ __forceinline__ int64_t end(int64_t b) const {
    bool bad;
    return end(b, bad);
  }
  // whether a compact list is worth forming
  __host__ __device__ __forceinline__ bool listed() const {
    return (window || rollout) && B <= kListMax && B * T < (int64_t(1) << 31);
  }
};

struct RowList {
  int32_t off[kListMax + 1];   // exclusive prefix sums of the processed ranges

  // All threads of the CTA; ends with a barrier.  CTA 0 reports invalid lengths.
  __device__ __forceinline__ void build(const RowRange& r, int32_t* status) {
    if (!r.listed()) {
      if ((r.window || r.rollout) && blockIdx.x == 0) {
        for (int64_t b = threadIdx.x; b < r.B; b += blockDim.x) {
          bool bad;
          r.end(b, bad);
          if (bad) atomicOr(status, (int32_t)ADWIN_DEV_WINDOW);
        }
      }
      __syncthreads();
      return;
    }
    const int n = (int)r.B;
    for (int b = threadIdx.x; b < n; b += blockDim.x) {
      bool bad;
      off[b + 1] = (int32_t)r.end(b, bad);
      if (bad && blockIdx.x == 0) atomicOr(status, (int32_t)ADWIN_DEV_WINDOW);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      int run = 0;
      for (int b0 = 0; b0 < n; b0 += 32) {
        const int b = b0 + (int)threadIdx.x;
        int v = b < n ? off[b + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, v, o);
          if ((int)threadIdx.x >= o) v += u;
        }
        if (b < n) off[b + 1] = run + v;
        run += __shfl_sync(0xffffffffu, v, 31);
      }
      if (threadIdx.x == 0) off[0] = 0;
    }
    __syncthreads();
  }
  __device__ __forceinline__ int64_t count(const RowRange& r) const {
    return r.listed() ? (int64_t)off[r.B] : r.B * r.T;
  }
  // Position of the n-th row of the list, or -1: a position outside its sequence's range.
  __device__ __forceinline__ int64_t row(const RowRange& r, int64_t n) const {
    if (!r.listed()) {
      if (!r.window && !r.rollout) return n;
      const int64_t b = n / r.T;
      return n - b * r.T < r.end(b) ? n : -1;
    }
    int lo = 0, hi = (int)r.B;   // off[lo] <= n < off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (off[mid] <= (int)n) lo = mid; else hi = mid;
    }
    return (int64_t)lo * r.T + (n - off[lo]);
  }
};

// Calls f(r) for the positions outside the processed ranges, spread over all threads of the grid.
template <typename F>
__device__ __forceinline__ void for_rows_outside(const RowRange& r, const RowList& list, F f) {
  if ((!r.window && !r.rollout) || (r.listed() && list.count(r) == r.B * r.T)) return;
  const int64_t rows = r.B * r.T, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows; i += step) {
    const int64_t b = i / r.T;
    if (i - b * r.T >= r.end(b)) f(i);
  }
}

// Zero-fills the gradient rows outside the processed ranges, a warp per row.
template <typename TOut>
__device__ __forceinline__ void zero_rows_outside(const RowRange& r, void* grad, int64_t ld, int64_t V) {
  if (!r.window && !r.rollout) return;
  const int64_t rows = r.B * r.T, warps = (int64_t)gridDim.x * (blockDim.x >> 5);
  const int lane = threadIdx.x & 31;
  for (int64_t i = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < rows; i += warps) {
    const int64_t b = i / r.T;
    if (i - b * r.T < r.end(b)) continue;
    TOut* g = static_cast<TOut*>(grad) + i * ld;
    constexpr int N = 16 / sizeof(TOut);
    int64_t head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / (int64_t)sizeof(TOut);
    if (head > V) head = V;
    const int64_t pieces = (V - head) / N, tail = V - head - pieces * N;
    if (lane < head) g[lane] = TOut(0.f);
    if (lane < tail) g[V - tail + lane] = TOut(0.f);
    uint4* o = reinterpret_cast<uint4*>(g + head);
    for (int64_t k = lane; k < pieces; k += 32) __stcs(o + k, make_uint4(0u, 0u, 0u, 0u));
  }
}

// How a row lies in memory: `head` entries up to the first 16-byte boundary, whole 16-byte pieces,
// `tail` entries.  Rows of a few entries are all head.
struct RowPieces {
  int head, tail;
  int64_t pieces;
  template <typename TIn>
  __device__ static __forceinline__ RowPieces of(const void* row, int64_t V) {
    constexpr int N = Elem<TIn>::N;
    RowPieces p;
    if (V < 4 * N) {
      p.head = (int)V;
      p.tail = 0;
      p.pieces = 0;
      return p;
    }
    p.head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(TIn);
    p.pieces = (V - p.head) / N;
    p.tail = (int)(V - p.head - p.pieces * N);
    return p;
  }
};

}  // namespace adwin
