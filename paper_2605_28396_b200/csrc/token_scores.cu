// Scores of given tokens under one policy: log probability, entropy, log-sum-exp, the K most likely
// alternatives and the mass outside them; and the gradient of any loss of these scores.
//
// token_scores_kernel, one row (or a slice of it, see below) per CTA, read once:
//   lse = M + ln S,  S = sum e^(z-M);   H = ln S + (sum e^(z-M) (M-z)) / S   (terms of one sign);
//   logprob = (z_y - M) - ln S, so that nothing of the size of M is rounded into it.
// Sums are formed in fp32 against the maximum of each thread's group of eight 16-byte loads and
// merged by weights 2^(m - m'), so there is no second read and no entry, however low or masked, that
// a reference could lose.
//
// The alternatives come from the same sweep.  A thread writes down, for each `unit` of a few groups
// of loads, the largest logit and the sum of exponentials.  The K-th largest of the units' maxima, tau, is a lower
// bound of the K-th largest entry, so only units whose maximum reaches tau hold alternatives: about
// K of them, a few KB that are still in L2.  Their entries >= tau, about K again, are ranked against one
// another (larger first, then lower index).  The mass outside is the sum over the units that were
// not opened, the entries below tau in those that were, and the losers: all terms positive, so it
// keeps its relative precision however small it is (as 1 - sum of the list it would not).  A row with
// more than kCand entries >= tau (long ties, sorted rows) has its threshold found by bisection, on
// the value and then on the index, over the opened units.  Nothing depends on the order of atomics:
// the candidates' ranks do not, and sums run in the order of ranks and units.
//
// token_scores_bwd_kernel: g_k = p_k (c0 + c1 log p_k) + what the entry has of its own
// (d_logprob at the token, d_top at the alternatives), one read and one write per entry; the few
// entries of the second kind are written again once the slice is done.
#include "adwin_common.cuh"
#include "adwin_internal.h"
#include "exp_sums.cuh"
#include "row_list.cuh"

namespace adwin {
namespace {

constexpr int kUnroll = 8;       // 16-byte loads in flight per thread
constexpr int kSlots = 12;       // units of a thread, at most
constexpr int kCand = 384;       // entries that can be ranked at once
constexpr int kMaxClusterX = 8;
// Order of floats as order of whole numbers, and back.
__device__ __forceinline__ int order_key(float z) {
  const int b = __float_as_int(z + 0.f);
  return b >= 0 ? b : b ^ 0x7fffffff;
}
__device__ __forceinline__ float key_value(int k) { return __int_as_float(k >= 0 ? k : k ^ 0x7fffffff); }

// Sum of exponentials against a finite reference m: s = sum 2^t, a = sum t 2^t, t = (z - m) log2 e.
struct ExpSum {
  float m, s, a;
  __device__ __forceinline__ void reset() {
    m = kLowest;
    s = a = 0.f;
  }
  __device__ __forceinline__ void merge(const ExpSum& x) {
    const float nm = fmaxf(m, x.m);
    const float t0 = max_nan((m - nm) * kLog2e, kNil), t1 = max_nan((x.m - nm) * kLog2e, kNil);
    const float w0 = ex2f(t0), w1 = ex2f(t1);
    a = w0 * fmaf(s, t0, a) + w1 * fmaf(x.s, t1, x.a);
    s = fmaf(w0, s, w1 * x.s);
    m = nm;
  }
};

// The mass outside the list, against its own largest entry: it may be far below what the row's sum
// can resolve, and below the smallest fp32 number relative to the row's maximum.
struct Mass {
  float m, s;
  __device__ __forceinline__ void add(float zm, float zs) {   // zs >= 0 against zm
    const float nm = fmaxf(m, zm);
    s = fmaf(ex2f(max_nan((m - nm) * kLog2e, kNil)), s, ex2f(max_nan((zm - nm) * kLog2e, kNil)) * zs);
    m = nm;
  }
  __device__ __forceinline__ void add(float z) {
    if (z > m) {
      s = fmaf(ex2f(max_nan((m - z) * kLog2e, kNil)), s, 1.f);
      m = z;
    } else {   // (-inf adds nothing, also against the lowest value that an empty mass refers to)
      s += ex2f(max_nan((z - m) * kLog2e, kNil));
    }
  }
};

// 2^((z - m) log2 e) and its exponent of a pair.  The difference is formed first, so that an entry at
// the reference has the exponent 0 whatever its size; masked entries (-inf, the lowest value) end
// at kNil, where the exponential is zero and the product with it too; NaN stays.
__device__ __forceinline__ f2_t exponent2(f2_t z, f2_t neg_m) {
  float tl, th;
  upk2(mul2(add2(z, neg_m), splat2(kLog2e)), tl, th);
  return pk2(max_nan(tl, kNil), max_nan(th, kNil));
}

template <typename TIn, int U>
__device__ __forceinline__ ExpSum group_sum(const uint4 (&v)[U], float gmax) {
  ExpSum g;
  g.m = fmaxf(gmax, kLowest);
  const f2_t neg_m = splat2(-g.m);
  f2_t S = 0ull, A = 0ull;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    f2_t z[Pairs<TIn>::NP];
    Pairs<TIn>::make(v[k], z);
#pragma unroll
    for (int j = 0; j < Pairs<TIn>::NP; ++j) {
      const f2_t t = exponent2(z[j], neg_m), e = ex2_2(t);
      S = add2(S, e);
      A = fma2(e, t, A);
    }
  }
  g.s = hsum2(S);
  g.a = hsum2(A);
  return g;
}

struct ScoreParams {
  const void* logits;
  int64_t V, ld;
  RowRange range;
  const int32_t* tokens;
  int K;
  float *logprob, *entropy, *lse;   // entropy, lse: may be null
  int32_t* top_ids;
  float *top_logprobs, *rest;       // rest: may be null
  int32_t* status;
};

// What a CTA of a cluster hands to the first one.
struct alignas(16) SliceResult {
  float m, s, a;
  Mass rest;
  int n;                 // entries of its list
  int pad[2];
  float z[ADWIN_TOP_MAX];
  int32_t id[ADWIN_TOP_MAX];
};

template <int TH>
struct ScoreShared {
  RowList list;
  float red[3][TH / 32];
  int count[2][TH / 32];
  int low[TH / 32], high[TH / 32];
  int n_cand;
  // alternatives
  float unit_sum[kSlots * TH];
  int unit_key[kSlots * TH];
  uint16_t open[kSlots * TH];
  float cand_z[kCand];
  int32_t cand_id[kCand];
  float sorted_z[kCand];
  int32_t sorted_id[kCand];
};

// Sum over the CTA of a whole number per thread, one barrier; consecutive calls alternate `flip`.
template <int TH>
__device__ __forceinline__ int block_count(int v, int (&slots)[2][TH / 32], int& flip) {
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) slots[flip][threadIdx.x >> 5] = v;
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) n += slots[flip][w];
  flip ^= 1;
  return n;
}

// Mass over the CTA of one per thread, in a fixed order; every thread returns it.
template <int TH>
__device__ __forceinline__ Mass block_mass(Mass v, float (&m)[TH / 32], float (&s)[TH / 32]) {
  const float wm = warp_max(v.m);
  const float ws = lane_sum(ex2f(max_nan((v.m - wm) * kLog2e, kNil)) * v.s);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
    m[threadIdx.x >> 5] = wm;
    s[threadIdx.x >> 5] = ws;
  }
  __syncthreads();
  Mass t = {kLowest, 0.f};
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) t.add(m[w], s[w]);
  return t;
}

// A CTA's slice of a row.
template <typename TIn>
struct Slice {
  const char* row;
  const uint4* src;      // first piece of the slice
  int64_t entry0;        // vocabulary index of its first entry
  int64_t np;            // pieces
  int groups;            // groups of loads per unit
  int64_t edge;          // an entry beside the pieces that this thread holds, or -1
  float edge_z;
};

// Walks the pieces of the opened units and this thread's edge entry: f(z, index) per entry.
template <typename TIn, int TH, typename F>
__device__ __forceinline__ void for_opened(const Slice<TIn>& s, const uint16_t* open, int n_open,
                                           int32_t* status, F f) {
  constexpr int N = Elem<TIn>::N;
  const int per = s.groups * kUnroll, total = n_open * per;
  constexpr int kBatch = 4;
  for (int i0 = threadIdx.x; i0 < total; i0 += kBatch * TH) {
    uint4 v[kBatch];
    int64_t piece[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * TH;
      piece[q] = -1;
      if (i < total) {
        const int u = open[i / per], w = i % per;
        const int64_t p = ((int64_t)(u / TH) * s.groups + w / kUnroll) * (kUnroll * TH) +
                          (w % kUnroll) * TH + (u % TH);
        if (p < s.np && ADWIN_CHK(u < kSlots * TH, status)) {
          piece[q] = p;
          v[q] = __ldcg(s.src + p);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (piece[q] < 0) continue;
      float z[N];
      Elem<TIn>::unpack(v[q], z);
      const int64_t k0 = s.entry0 + piece[q] * N;
#pragma unroll
      for (int j = 0; j < N; ++j) f(z[j], k0 + j);
    }
  }
  if (s.edge >= 0) f(s.edge_z, s.edge);
}

// The K largest entries of the slice into sh.sorted_z / sorted_id (fewer if it has fewer); returns their number and the
// mass of all the others in `rest`.
template <typename TIn, int TH>
__device__ int select_top(ScoreShared<TH>& sh, const Slice<TIn>& s, int K, float M, int slots, int32_t* status,
                          Mass& rest) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int flip = 0;
  // a thread reads back its own units only
  int kmin = 0x7fffffff, kmax = (int)0x80000000, mine = 0;
  for (int j = 0; j < slots; ++j) {
    const int k = sh.unit_key[j * TH + tid];
    if (k == (int)0x80000000) continue;
    kmin = min(kmin, k);
    kmax = max(kmax, k);
    ++mine;
  }
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) {
    sh.low[warp] = kmin;
    sh.high[warp] = kmax;
  }
  if (tid == 0) sh.n_cand = 0;
  const int units = block_count<TH>(mine, sh.count, flip);
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) {
    kmin = min(kmin, sh.low[w]);
    kmax = max(kmax, sh.high[w]);
  }
  // tau: at least K units reach it, few more where the maxima differ
  int tau = (int)0x80000000;
  if (units > K) {
    int64_t lo = kmin, hi = (int64_t)kmax + 1;
    int c = units;
    const int enough = K + K / 4 + 4;
    while (hi - lo != 1 && c > enough) {
      const int64_t mid = lo + ((hi - lo) >> 1);
      int v = 0;
      for (int j = 0; j < slots; ++j) v += sh.unit_key[j * TH + tid] >= mid ? 1 : 0;
      const int n = block_count<TH>(v, sh.count, flip);
      if (n >= K) {
        lo = mid;
        c = n;
      } else {
        hi = mid;
      }
    }
    tau = (int)lo;
  }
  const float tau_z = tau == (int)0x80000000 ? -INFINITY : key_value(tau);
  // the opened units, in an order of their own; the others' sums
  Mass others = {kLowest, 0.f};
  int n_mine = 0;
  for (int j = 0; j < slots; ++j) {
    const int k = sh.unit_key[j * TH + tid];
    if (k == (int)0x80000000) continue;
    if (k >= tau) {
      ++n_mine;
    } else {
      others.add(fmaxf(key_value(k), kLowest), sh.unit_sum[j * TH + tid]);
    }
  }
  int before = n_mine;   // inclusive scan over the warp, then over the warps
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += u;
  }
  __syncthreads();   // (every thread has read sh.low)
  if (lane == 31) sh.low[warp] = before;
  __syncthreads();
  int n_open = 0, at = before - n_mine;
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) {
    if (w < warp) at += sh.low[w];
    n_open += sh.low[w];
  }
  for (int j = 0; j < slots; ++j) {
    const int k = sh.unit_key[j * TH + tid];
    if (k != (int)0x80000000 && k >= tau) sh.open[at++] = (uint16_t)(j * TH + tid);
  }
  __syncthreads();

  Mass below = {kLowest, 0.f};
  for_opened<TIn, TH>(s, sh.open, n_open, status, [&](float z, int64_t k) {
    if (z >= tau_z) {
      const int i = atomicAdd(&sh.n_cand, 1);
      if (i < kCand) {
        sh.cand_z[i] = z;
        sh.cand_id[i] = (int32_t)k;
      }
    } else {
      below.add(z);
    }
  });
  __syncthreads();
  int n = sh.n_cand;
  if (n > kCand) {
    // the K-th largest value by bisection between tau and the largest, then the index up to which
    // entries of that value belong to the list
    int64_t lo = tau == (int)0x80000000 ? order_key(-INFINITY) : tau, hi = (int64_t)order_key(M) + 1;
    int c = n;
    auto count = [&](float above, float equal, int64_t upto) {
      int v = 0;
      for_opened<TIn, TH>(s, sh.open, n_open, status, [&](float z, int64_t k) {
        v += (z >= above || (z >= equal && k <= upto)) ? 1 : 0;
      });
      return block_count<TH>(v, sh.count, flip);
    };
    while (hi - lo != 1 && c != K) {
      const int64_t mid = lo + ((hi - lo) >> 1);
      const int v = count(key_value((int)mid), INFINITY, -1);
      if (v >= K) {
        lo = mid;
        c = v;
      } else {
        hi = mid;
      }
    }
    const float equal = key_value((int)lo), above = c == K ? equal : key_value((int)hi);
    int64_t ilo = -1, ihi = s.entry0 + s.np * Elem<TIn>::N + Elem<TIn>::N;   // up to ilo: too few
    if (c != K) {
      while (ihi - ilo > 1) {
        const int64_t mid = (ilo + ihi) >> 1;
        if (count(above, equal, mid) >= K) ihi = mid; else ilo = mid;
      }
    }
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
    below = Mass{kLowest, 0.f};
    for_opened<TIn, TH>(s, sh.open, n_open, status, [&](float z, int64_t k) {
      if (z >= above || (z >= equal && k <= ihi)) {
        const int i = atomicAdd(&sh.n_cand, 1);
        if (ADWIN_CHK(i < kCand, status)) {
          sh.cand_z[i] = z;
          sh.cand_id[i] = (int32_t)k;
        }
      } else {
        below.add(z);
      }
    });
    __syncthreads();
    n = min(sh.n_cand, kCand);
  }
  for (int i = tid; i < n; i += TH) {
    const float z = sh.cand_z[i];
    const int32_t id = sh.cand_id[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) {
      const float x = sh.cand_z[j];
      rank += (x > z || (x == z && sh.cand_id[j] < id)) ? 1 : 0;
    }
    sh.sorted_z[rank] = z;
    sh.sorted_id[rank] = id;
  }
  __syncthreads();
  for (int i = K + tid; i < n; i += TH) below.add(sh.sorted_z[i]);
  below.add(others.m, others.s);
  rest = block_mass<TH>(below, sh.red[0], sh.red[1]);
  return n < K ? n : K;
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}

// TOP: alternatives are wanted.  Clusters: the CTAs of a cluster take a slice of the row each and
// the first one joins their sums and lists.
template <typename TIn, int TH, bool TOP>
__global__ void __launch_bounds__(TH, TH == 128 ? 8 : 1) token_scores_kernel(const ScoreParams p) {
  chain();
  extern __shared__ __align__(16) uint8_t smem[];
  ScoreShared<TH>& sh = *reinterpret_cast<ScoreShared<TH>*>(smem);
  constexpr size_t kOwn = TOP ? sizeof(ScoreShared<TH>) : offsetof(ScoreShared<TH>, unit_sum);
  SliceResult* slices = reinterpret_cast<SliceResult*>(smem + ((kOwn + 15) & ~size_t(15)));
  constexpr int N = Elem<TIn>::N;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = (int)cluster_size(), me = C > 1 ? (int)cluster_rank() : 0;
  const int K = TOP ? p.K : 0;

  sh.list.build(p.range, p.status);
  for_rows_outside(p.range, [&](int64_t r) {
    p.logprob[r] = 0.f;
    if (p.entropy) p.entropy[r] = 0.f;
    if (p.lse) p.lse[r] = 0.f;
    if (p.rest) p.rest[r] = 0.f;
    for (int j = 0; j < K; ++j) {
      p.top_ids[r * K + j] = -1;
      p.top_logprobs[r * K + j] = 0.f;
    }
  });

  if (C > 1) cluster_sync_all();   // every CTA is there before anything is written to one

  const int64_t rows = sh.list.count(p.range);
  for (int64_t n = blockIdx.x / C; n < rows; n += gridDim.x / C) {
    const int64_t r = sh.list.row(p.range, n);
    if (r < 0) continue;
    Slice<TIn> s;
    s.row = static_cast<const char*>(p.logits) + (size_t)r * p.ld * sizeof(TIn);
    const RowPieces rp = RowPieces::of<TIn>(s.row, p.V);
    const int64_t per = (rp.pieces + C - 1) / C, first = per * me < rp.pieces ? per * me : rp.pieces;
    s.np = first + per < rp.pieces ? per : rp.pieces - first;
    s.entry0 = rp.head + first * N;
    s.src = reinterpret_cast<const uint4*>(s.row + (size_t)s.entry0 * sizeof(TIn));
    s.edge = -1;
    if (me == 0 && tid < rp.head) s.edge = tid;
    if (me == C - 1 && tid >= 32 && tid - 32 < rp.tail) s.edge = p.V - rp.tail + (tid - 32);
    s.edge_z = s.edge >= 0 ? Elem<TIn>::load1(s.row, s.edge) : 0.f;
    const int64_t trips = (s.np + kUnroll * TH - 1) / (kUnroll * TH);
    s.groups = (int)((trips + kSlots - 1) / kSlots);
    if (s.groups < 1) s.groups = 1;
    const int slots = (int)((trips + s.groups - 1) / s.groups);
    const int y = (me == 0 && tid == 0) ? p.tokens[r] : 0;
    const bool y_valid = y >= 0 && (int64_t)y < p.V;
    const float zy = (me == 0 && tid == 0 && y_valid) ? Elem<TIn>::load1(s.row, y) : 0.f;

    ExpSum acc;
    acc.reset();
    if (s.edge >= 0) {
      acc.m = fmaxf(s.edge_z, kLowest);
      const float t = max_nan((s.edge_z - acc.m) * kLog2e, kNil);
      acc.s = ex2f(t);
      acc.a = acc.s * t;
    }
    int64_t i = tid;
    for (int slot = 0; slot < slots; ++slot) {
      ExpSum unit;
      unit.reset();
      int key = (int)0x80000000;
      for (int g = 0; g < s.groups; ++g, i += kUnroll * TH) {
        if (i - tid >= s.np) break;
        uint4 v[kUnroll];
        if (i - tid + kUnroll * TH <= s.np) {
#pragma unroll
          for (int k = 0; k < kUnroll; ++k)
            if (ADWIN_CHK(s.entry0 + (i + k * TH + 1) * N <= p.V, p.status)) v[k] = __ldcs(s.src + i + k * TH);
        } else {
          constexpr uint32_t kMasked = sizeof(TIn) == 2 ? 0xff80ff80u : 0xff800000u;   // -infinity
#pragma unroll
          for (int k = 0; k < kUnroll; ++k) {
            v[k] = make_uint4(kMasked, kMasked, kMasked, kMasked);
            if (i + k * TH < s.np && ADWIN_CHK(s.entry0 + (i + k * TH + 1) * N <= p.V, p.status))
              v[k] = __ldcs(s.src + i + k * TH);
          }
        }
        const float gm = group_max(v, static_cast<TIn*>(nullptr));
        if (TOP && i < s.np) key = max(key, order_key(gm));
        unit.merge(group_sum<TIn, kUnroll>(v, gm));
      }
      if (TOP) {
        sh.unit_key[slot * TH + tid] = key;
        sh.unit_sum[slot * TH + tid] = unit.s;
      }
      acc.merge(unit);
    }
    // the CTA's sum, in a fixed order
    ExpSum tot;
    {
      const float wm = warp_max(acc.m);
      const float t = max_nan((acc.m - wm) * kLog2e, kNil), w = ex2f(t);
      const float ws = lane_sum(w * acc.s), wa = lane_sum(w * fmaf(acc.s, t, acc.a));
      if (lane == 0) {
        sh.red[0][warp] = wm;
        sh.red[1][warp] = ws;
        sh.red[2][warp] = wa;
      }
      __syncthreads();
      tot.reset();
#pragma unroll
      for (int q = 0; q < TH / 32; ++q) tot.m = fmaxf(tot.m, sh.red[0][q]);
#pragma unroll
      for (int q = 0; q < TH / 32; ++q) {
        const float tq = max_nan((sh.red[0][q] - tot.m) * kLog2e, kNil), wq = ex2f(tq);
        tot.s = fmaf(wq, sh.red[1][q], tot.s);
        tot.a = fmaf(wq, fmaf(sh.red[1][q], tq, sh.red[2][q]), tot.a);
      }
    }
    // (a slice of masked entries only is no reason to stop, a NaN or +infinity is)
    const bool sound = isfinite(tot.s) && isfinite(tot.m);
    Mass rest = {kLowest, 0.f};
    int n_top = 0;
    if (TOP && sound && (C > 1 || tot.s > 0.f))
      n_top = select_top<TIn, TH>(sh, s, K, tot.m, slots, p.status, rest);

    const float* list_z = TOP ? sh.sorted_z : nullptr;
    const int32_t* list_id = TOP ? sh.sorted_id : nullptr;
    if (C > 1) {
      // hand the slice's result to the first CTA
      const uint32_t dst = map_to_rank(smem_u32(&slices[me]), 0);
      if (tid == 0) {
        remote_store4(dst, tot.m, tot.s, tot.a, rest.m);
        remote_store4(dst + 16, rest.s, __int_as_float(n_top), 0.f, 0.f);
      }
      if (TOP && tid < n_top) {
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + (uint32_t)offsetof(SliceResult, z) + 4 * tid),
                     "f"(sh.sorted_z[tid]) : "memory");
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(dst + (uint32_t)offsetof(SliceResult, id) + 4 * tid),
                     "r"(sh.sorted_id[tid]) : "memory");
      }
      cluster_sync_all();
      if (me == 0) {
        tot.reset();
        for (int q = 0; q < C; ++q) tot.m = fmaxf(tot.m, slices[q].m);
        rest = Mass{kLowest, 0.f};
        for (int q = 0; q < C; ++q) {
          const float tq = max_nan((slices[q].m - tot.m) * kLog2e, kNil), wq = ex2f(tq);
          tot.s = fmaf(wq, slices[q].s, tot.s);
          tot.a = fmaf(wq, fmaf(slices[q].s, tq, slices[q].a), tot.a);
          rest.add(slices[q].rest.m, slices[q].rest.s);
        }
        if constexpr (TOP) {
          // rank of an entry: its place in its own list and, by bisection, in the others'; equal
          // entries of an earlier slice come first, they have the lower index
          Mass losers = {kLowest, 0.f};
          for (int i2 = tid; i2 < C * K; i2 += TH) {
            const int q = i2 / K, j = i2 % K;
            if (j >= slices[q].n) continue;
            const float z = slices[q].z[j];
            int rank = j;
            for (int o = 0; o < C; ++o) {
              if (o == q) continue;
              int lo = 0, hi = slices[o].n;
              while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                const float x = slices[o].z[mid];
                if (x > z || (x == z && o < q)) lo = mid + 1; else hi = mid;
              }
              rank += lo;
            }
            if (rank < K) {
              sh.cand_z[rank] = z;
              sh.cand_id[rank] = slices[q].id[j];
            } else {
              losers.add(z);
            }
          }
          losers = block_mass<TH>(losers, sh.red[0], sh.red[1]);   // (its barriers publish the list)
          rest.add(losers.m, losers.s);
          list_z = sh.cand_z;
          list_id = sh.cand_id;
        }
      }
    }
    if (me == 0) {
      const float ln_s = logf(tot.s), lse = tot.m + ln_s;
      const bool finite = isfinite(lse);
      const float nan = __int_as_float(0x7fc00000);
      if constexpr (TOP) {
        for (int j = tid; j < K; j += TH) {
          p.top_ids[r * K + j] = finite ? list_id[j] : -1;
          p.top_logprobs[r * K + j] = finite ? (list_z[j] - tot.m) - ln_s : nan;
        }
      }
      if (tid == 0) {
        p.logprob[r] = (y_valid && finite) ? (zy - tot.m) - ln_s : nan;
        if (p.entropy) p.entropy[r] = finite ? fmaf(-tot.a / tot.s, kLn2, ln_s) : nan;
        if (p.lse) p.lse[r] = lse;
        if (p.rest) p.rest[r] = finite ? (rest.m - tot.m) + (logf(rest.s) - ln_s) : nan;
        int bits = 0;
        if (!y_valid) bits |= ADWIN_DEV_TOKEN_RANGE;
        if (!finite) bits |= ADWIN_DEV_NONFINITE;
        if (bits) atomicOr(p.status, bits);
      }
    }
    if (C > 1) cluster_sync_all(); else __syncthreads();   // before the next row overwrites anything
  }
}

// ---------------------------------------------------------------------------- gradient
struct ScoreBwdParams {
  const void* logits;
  int64_t V, ld;
  RowRange range;
  const int32_t* tokens;
  const float *lse, *entropy, *d_logprob, *d_entropy;   // entropy, d_*: may be null
  const int32_t* top_ids;
  const float* d_top;
  int K;
  int splits;          // CTAs per row
  bool zero_tail;
  void* grad;
  int64_t ld_grad;
  int32_t* status;
};

constexpr int kBwdThreads = 256;
constexpr int kBwdUnroll = 4;

template <typename TIn, typename TOut>
__global__ void __launch_bounds__(kBwdThreads, 4) token_scores_bwd_kernel(const ScoreBwdParams p) {
  chain();
  __shared__ RowList list;
  __shared__ int32_t own_id[ADWIN_TOP_MAX + 1];
  __shared__ float own_w[ADWIN_TOP_MAX + 1];
  __shared__ float sum_w;
  __shared__ int any;
  constexpr int N = Elem<TIn>::N, NP = Pairs<TIn>::NP;
  const int tid = threadIdx.x;
  list.build(p.range, p.status);
  const int64_t items = list.count(p.range) * p.splits;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t r = list.row(p.range, item / p.splits);
    if (r < 0) continue;
    const int part = (int)(item % p.splits);
    const char* row = static_cast<const char*>(p.logits) + (size_t)r * p.ld * sizeof(TIn);
    char* out = static_cast<char*>(p.grad) + (size_t)r * p.ld_grad * sizeof(TOut);
    const RowPieces rp = RowPieces::of<TIn>(row, p.V);
    const int64_t per = (rp.pieces + p.splits - 1) / p.splits;
    const int64_t first = per * part < rp.pieces ? per * part : rp.pieces;
    const int64_t np = first + per < rp.pieces ? per : rp.pieces - first;
    const int64_t entry0 = rp.head + first * N;
    const bool last = part == p.splits - 1;
    // entries of the slice: [begin, end), and the tail in the last one
    const int64_t begin = part == 0 ? 0 : entry0, end = last ? p.V : entry0 + np * N;

    // weights of single entries: the alternatives', the token's behind them
    if (tid <= p.K) {
      int32_t id = -1;
      float w = 0.f;
      if (tid < p.K) {
        id = p.top_ids[r * p.K + tid];
        w = p.d_top[r * p.K + tid];
      } else if (p.d_logprob) {
        id = p.tokens[r];
        w = p.d_logprob[r];
        if (id == -1) id = -2;   // (a token has no "none")
      }
      if (id < 0 || (int64_t)id >= p.V) {
        if (id != -1 && part == 0) atomicOr(p.status, (int32_t)ADWIN_DEV_TOKEN_RANGE);
        id = -1;
        w = 0.f;
      }
      own_id[tid] = id;
      own_w[tid] = w;
    }
    __syncthreads();
    const float h = p.d_entropy ? p.d_entropy[r] : 0.f;
    if (tid < 32) {
      float w = 0.f;
      bool some = h != 0.f;
      for (int j = tid; j <= p.K; j += 32) {
        w += own_w[j];
        some = some || own_w[j] != 0.f;
      }
      w = lane_sum(w);
      some = __any_sync(0xffffffffu, some);
      if (tid == 0) {
        sum_w = w;
        any = some;
      }
    }
    // this thread's single entry, read before the gradient may overwrite it (grad may be the logits)
    const int64_t mine = tid <= p.K ? own_id[tid] : -1;
    const bool patch = mine >= begin && mine < end;   // (none: -1)
    const float z_mine = patch ? Elem<TIn>::load1(row, mine) : 0.f;
    const int64_t edge = (part == 0 && tid < rp.head) ? tid
                         : (last && tid >= 32 && tid - 32 < rp.tail) ? p.V - rp.tail + (tid - 32) : -1;
    const float z_edge = edge >= 0 ? Elem<TIn>::load1(row, edge) : 0.f;
    __syncthreads();

    const float lse = p.lse[r];
    // without any weight the row's gradient is zero whatever its logits
    const bool zero = !any;
    // g = p (c0 + c1 t), t = log2 p
    const float c0 = h != 0.f ? -fmaf(h, p.entropy[r], sum_w) : -sum_w, c1 = -h * kLn2;
    const f2_t neg_lse = splat2(-lse), C0 = splat2(c0), C1 = splat2(c1);
    auto grad1 = [&](float z) {
      const float t = max_nan((z - lse) * kLog2e, kNil);
      return zero ? 0.f : ex2f(t) * fmaf(c1, t, c0);
    };
    char* out0 = out + (size_t)entry0 * sizeof(TOut);
    constexpr int kOutAlign = N * sizeof(TOut) < 16 ? (int)(N * sizeof(TOut)) : 16;
    const bool wide = (reinterpret_cast<uintptr_t>(out0) & (kOutAlign - 1)) == 0;
    const uint4* src = reinterpret_cast<const uint4*>(row + (size_t)entry0 * sizeof(TIn));
    for (int64_t i = tid; i < np; i += kBwdUnroll * kBwdThreads) {
      uint4 v[kBwdUnroll];
#pragma unroll
      for (int k = 0; k < kBwdUnroll; ++k)
        if (!zero && i + k * kBwdThreads < np &&
            ADWIN_CHK(entry0 + (i + k * kBwdThreads + 1) * N <= p.V, p.status))
          v[k] = __ldcs(src + i + k * kBwdThreads);
#pragma unroll
      for (int k = 0; k < kBwdUnroll; ++k) {
        const int64_t q = i + k * kBwdThreads;
        if (q >= np) break;
        f2_t g[NP];
        if (zero) {
#pragma unroll
          for (int j = 0; j < NP; ++j) g[j] = 0ull;
        } else {
          f2_t z[NP];
          Pairs<TIn>::make(v[k], z);
#pragma unroll
          for (int j = 0; j < NP; ++j) {
            const f2_t t = exponent2(z[j], neg_lse);
            g[j] = mul2(ex2_2(t), fma2(C1, t, C0));
          }
        }
        if (wide) {
          store_pairs<TOut>(out0 + (size_t)q * N * sizeof(TOut), g);
        } else {
#pragma unroll
          for (int j = 0; j < NP; ++j) {
            float a, b;
            upk2(g[j], a, b);
            Elem<TOut>::store1(out0, q * N + 2 * j, a);
            Elem<TOut>::store1(out0, q * N + 2 * j + 1, b);
          }
        }
      }
    }
    if (edge >= 0) Elem<TOut>::store1(out, edge, grad1(z_edge));
    __syncthreads();   // the patches come after the sweep's stores
    if (patch) {
      float g = grad1(z_mine);
      for (int j = 0; j <= p.K; ++j) g += own_id[j] == (int32_t)mine ? own_w[j] : 0.f;
      if (ADWIN_CHK(mine < p.V, p.status)) Elem<TOut>::store1(out, mine, g);
    }
    __syncthreads();
  }
  if (p.zero_tail) zero_rows_outside<TOut>(p.range, p.grad, p.ld_grad, p.V);
}

template <typename TIn, int TH, bool TOP>
cudaError_t launch_scores(const ScoreParams& p, int64_t clusters, int C, cudaStream_t s) {
  size_t smem = TOP ? sizeof(ScoreShared<TH>) : offsetof(ScoreShared<TH>, unit_sum);
  smem = (smem + 15) & ~size_t(15);
  // (one limit for every launch of this kernel: launches of other threads may come in between)
  constexpr size_t limit = sizeof(ScoreShared<TH>) + 16 + kMaxClusterX * sizeof(SliceResult);
  if (C > 1) smem += C * sizeof(SliceResult);
  const cudaError_t e = cudaFuncSetAttribute(token_scores_kernel<TIn, TH, TOP>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, (int)limit);
  if (e != cudaSuccess) return e;
  return launch_chained(token_scores_kernel<TIn, TH, TOP>, (unsigned)(clusters * C), TH, smem, C, s, p);
}

}  // namespace

cudaError_t launch_token_scores(const void* logits, int dtype, int64_t B, int64_t T, int64_t V, int64_t ld,
                                const int32_t* tokens, const int32_t* window, const int32_t* rollout_len,
                                int K, float* logprob, float* entropy, float* lse, int32_t* top_ids,
                                float* top_logprobs, float* rest, int32_t* status, int sm_count,
                                cudaStream_t s) {
  ScoreParams p = {};
  p.logits = logits;
  p.V = V;
  p.ld = ld;
  p.range = RowRange{window, rollout_len, B, T};
  p.tokens = tokens;
  p.K = K;
  p.logprob = logprob;
  p.entropy = entropy;
  p.lse = lse;
  p.top_ids = top_ids;
  p.top_logprobs = top_logprobs;
  p.rest = K > 0 ? rest : nullptr;
  p.status = status;
  const int64_t rows = B * T;
  const bool bf = dtype == ADWIN_BF16;
  const int64_t pieces = V / (bf ? 8 : 4);
  // few rows: clusters of CTAs with 512 threads share a row, so that the call reads with the whole GPU
  int C = 1;
  while (C < kMaxClusterX && rows * C * 2 <= sm_count && pieces >= (int64_t)C * 2 * 512) C *= 2;
  if (C > 1) {
#define ADWIN_SCORES(TOP) \
  (bf ? launch_scores<__nv_bfloat16, 512, TOP>(p, rows, C, s) : launch_scores<float, 512, TOP>(p, rows, C, s))
    return K > 0 ? ADWIN_SCORES(true) : ADWIN_SCORES(false);
#undef ADWIN_SCORES
  }
  int64_t grid = (int64_t)sm_count * 64;
  if (grid > rows) grid = rows;
#define ADWIN_SCORES(TOP) \
  (bf ? launch_scores<__nv_bfloat16, 128, TOP>(p, grid, 1, s) : launch_scores<float, 128, TOP>(p, grid, 1, s))
  return K > 0 ? ADWIN_SCORES(true) : ADWIN_SCORES(false);
#undef ADWIN_SCORES
}

cudaError_t launch_token_scores_bwd(const void* logits, int dtype, int64_t B, int64_t T, int64_t V, int64_t ld,
                                    const int32_t* tokens, const int32_t* window, const int32_t* rollout_len,
                                    const float* lse, const float* entropy, const float* d_logprob,
                                    const float* d_entropy, const int32_t* top_ids, const float* d_top, int K,
                                    int flags, void* grad, int grad_dtype, int64_t ld_grad, int32_t* status,
                                    int sm_count, cudaStream_t s) {
  ScoreBwdParams p = {};
  p.logits = logits;
  p.V = V;
  p.ld = ld;
  p.range = RowRange{window, rollout_len, B, T};
  p.tokens = tokens;
  p.lse = lse;
  p.entropy = entropy;
  p.d_logprob = d_logprob;
  p.d_entropy = d_entropy;
  p.top_ids = top_ids;
  p.d_top = d_top;
  p.K = d_top ? K : 0;
  p.zero_tail = (flags & ADWIN_ZERO_TAIL) != 0;
  p.grad = grad;
  p.ld_grad = ld_grad;
  p.status = status;
  const int64_t rows = B * T;
  const bool bf = dtype == ADWIN_BF16;
  // few rows are cut into slices of at least two rounds of loads
  const int64_t pieces = V / (bf ? 8 : 4), room = (int64_t)sm_count * 8;
  int64_t splits = 1;
  while (rows * splits * 2 <= room && pieces >= splits * 4 * kBwdUnroll * kBwdThreads) splits *= 2;
  p.splits = (int)splits;
  int64_t grid = (int64_t)sm_count * 32;
  if (grid > rows * splits) grid = rows * splits;
#define ADWIN_BWD(TIN, TOUT) \
  launch_chained(token_scores_bwd_kernel<TIN, TOUT>, (unsigned)grid, kBwdThreads, 0, 1, s, p)
  if (bf) return grad_dtype == ADWIN_BF16 ? ADWIN_BWD(__nv_bfloat16, __nv_bfloat16) : ADWIN_BWD(__nv_bfloat16, float);
  return grad_dtype == ADWIN_BF16 ? ADWIN_BWD(float, __nv_bfloat16) : ADWIN_BWD(float, float);
#undef ADWIN_BWD
}

}  // namespace adwin
