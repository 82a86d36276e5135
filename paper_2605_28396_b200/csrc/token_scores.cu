// Scores of given tokens under one policy: log probability, entropy, log-sum-exp, the K most likely
// alternatives and the mass outside them; and the gradient of a loss of the log probabilities and the entropy
// (lse and the mass outside carry none).
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
// keeps its relative precision however small it is (as 1 - sum of the list it would not); where the list holds less
// than half, its log is made of the list all the same: near 0 that has no rounding of the sums' size in it.  A row with
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
constexpr int kCand = 256;       // entries that can be ranked at once
constexpr int kMaxClusterX = 8;
constexpr int kNone = (int)0x80000000;   // below every order_key
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
  int K, units, groups;             // units: room for those of a CTA's slice; groups: of loads per unit
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
  int2 count[2][TH / 32];
  int low[TH / 32], high[TH / 32];
  int n_cand;
  // alternatives
  Mass rest;
  unsigned long long cand[kCand];    // rank_key
  int rank[kCand];
  float sorted_z[kCand];
  int32_t sorted_id[kCand];
};
// The units of a row of `slots` to a thread follow: no more than the call's rows need, for shared memory is
// taken from L1, where loads in flight wait (64 alternatives of 40 960 rows of 4 096 entries 1 037 us with room for 12 slots,
// 638 with 8, 631 with the one they need).
struct Units {
  float* sum;       // of exponentials, against the unit's largest logit
  int* key;         // order_key of that
  uint16_t* open;   // units that may hold alternatives
  static constexpr size_t kBytes = 10;   // per unit
};
// The CTA's shared memory.  The selection is not inlined (its registers would cost the sweep its own: 5 120 rows of
// 151 936 entries 580 us inlined; what lives across its call still spills at the 64 registers of eight CTAs per SM: 116 bytes
// stored and 140 read back per thread, bf16) and finds it by this name, not by a pointer that might lead anywhere.
extern __shared__ __align__(16) uint8_t score_smem[];
template <int TH>
__device__ __forceinline__ ScoreShared<TH>& score_shared() {
  return *reinterpret_cast<ScoreShared<TH>*>(score_smem);
}
template <int TH>
__host__ __device__ constexpr size_t units_offset() {
  return (sizeof(ScoreShared<TH>) + 15) & ~size_t(15);
}
template <int TH>
__device__ __forceinline__ Units units_of(int capacity) {
  Units u;
  u.sum = reinterpret_cast<float*>(score_smem + units_offset<TH>());
  u.key = reinterpret_cast<int*>(u.sum + capacity);
  u.open = reinterpret_cast<uint16_t*>(u.key + capacity);
  return u;
}

// Sums over the CTA of two whole numbers per thread, one barrier; consecutive calls alternate `flip`.
template <int TH>
__device__ __forceinline__ int2 block_count(int x, int y, int2 (&slots)[2][TH / 32], int& flip) {
  x = __reduce_add_sync(0xffffffffu, x);
  y = __reduce_add_sync(0xffffffffu, y);
  const int lane = threadIdx.x & 31;
  if (lane == 0) slots[flip][threadIdx.x >> 5] = make_int2(x, y);
  __syncthreads();
  int2 v = make_int2(0, 0);
  if (TH <= 128) {
#pragma unroll
    for (int w = 0; w < TH / 32; ++w) {
      v.x += slots[flip][w].x;
      v.y += slots[flip][w].y;
    }
  } else {
    if (lane < TH / 32) v = slots[flip][lane];
    v.x = __reduce_add_sync(0xffffffffu, v.x);
    v.y = __reduce_add_sync(0xffffffffu, v.y);
  }
  flip ^= 1;
  return v;
}

// Mass over the CTA of one per thread, in a fixed order; every thread returns it.
template <int TH>
__device__ __forceinline__ Mass block_mass(Mass v, float (&m)[TH / 32], float (&s)[TH / 32]) {
  const int lane = threadIdx.x & 31;
  const float wm = warp_max(v.m);
  const float ws = lane_sum(ex2f(max_nan((v.m - wm) * kLog2e, kNil)) * v.s);
  __syncthreads();
  if (lane == 0) {
    m[threadIdx.x >> 5] = wm;
    s[threadIdx.x >> 5] = ws;
  }
  __syncthreads();
  const float lm = lane < TH / 32 ? m[lane] : kLowest, ls = lane < TH / 32 ? s[lane] : 0.f;
  Mass t;
  t.m = warp_max(lm);
  t.s = lane_sum(ex2f(max_nan((lm - t.m) * kLog2e, kNil)) * ls);
  return t;
}

// Order of the alternatives as order of whole numbers: larger logits, then lower indices.
__device__ __forceinline__ unsigned long long rank_key(float z, int32_t id) {
  return ((unsigned long long)((uint32_t)order_key(z) ^ 0x80000000u) << 32) | (uint32_t)~id;
}
__device__ __forceinline__ float rank_logit(unsigned long long k) { return key_value((int)((uint32_t)(k >> 32) ^ 0x80000000u)); }
__device__ __forceinline__ int32_t rank_id(unsigned long long k) { return (int32_t)~(uint32_t)k; }

// A CTA's slice of a row.
template <typename TIn>
struct Slice {
  const char* row;
  const uint4* src;      // first piece of the slice
  int entry0;            // vocabulary index of its first entry
  int np;                // pieces
  int groups;            // groups of loads per unit
  int edge;              // an entry beside the pieces that this thread holds, or -1
  float edge_z;
};

// Walks the pieces of the opened units: f(piece, index of its first entry).
template <typename TIn, int TH, typename F>
__device__ __forceinline__ void for_opened(const Slice<TIn>& s, const uint16_t* open, int n_open,
                                           int32_t* status, F f) {
  constexpr int N = Elem<TIn>::N;
  const int per = s.groups * kUnroll, total = n_open * per;
  constexpr int kBatch = 1;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < total; i0 += kBatch * TH) {
    uint4 v[kBatch];
    int piece[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const uint32_t i = (uint32_t)(i0 + q * TH);
      piece[q] = -1;
      if (i < (uint32_t)total) {
        const uint32_t nth = s.groups == 1 ? i / kUnroll : i / (uint32_t)per;
        const int u = open[nth], w = (int)(i - nth * (uint32_t)per);
        const int p = ((u / TH) * s.groups + w / kUnroll) * (kUnroll * TH) + (w % kUnroll) * TH + (u % TH);
        if (p < s.np && ADWIN_CHK(u < kSlots * TH, status)) {
          piece[q] = p;
          v[q] = __ldcg(s.src + p);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (piece[q] >= 0) f(v[q], s.entry0 + piece[q] * N);
  }
}

// A piece's entries at and above a threshold: one bit each; the others stay, these become -inf.
__device__ __forceinline__ uint32_t split_piece(uint4& v, float from, __nv_bfloat16*) {
  const __nv_bfloat162 f2 = __float2bfloat162_rn(from);   // (a threshold is a value of the logits' type, or below all of them)
  uint32_t w[4] = {v.x, v.y, v.z, v.w}, bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = __hge2_mask(reinterpret_cast<const __nv_bfloat162&>(w[i]), f2);
    bits |= (m & (1u << (2 * i))) | (m & (2u << (2 * i + 16))) >> 16;
    w[i] = (w[i] & ~m) | (0xff80ff80u & m);
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
  return bits;
}
__device__ __forceinline__ uint32_t split_piece(uint4& v, float from, float*) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w}, bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool in = __uint_as_float(w[i]) >= from;
    bits |= (in ? 1u : 0u) << i;
    if (in) w[i] = 0xff800000u;
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
  return bits;
}
// Their number alone.
__device__ __forceinline__ int count_piece(const uint4& v, float from, __nv_bfloat16*) {
  const __nv_bfloat162 f2 = __float2bfloat162_rn(from);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t n = 0;   // per half
#pragma unroll
  for (int i = 0; i < 4; ++i) n += __hge2_mask(reinterpret_cast<const __nv_bfloat162&>(w[i]), f2) & 0x00010001u;
  return (int)((n & 0xffffu) + (n >> 16));
}
__device__ __forceinline__ int count_piece(const uint4& v, float from, float*) {
  return (__uint_as_float(v.x) >= from) + (__uint_as_float(v.y) >= from) + (__uint_as_float(v.z) >= from) +
         (__uint_as_float(v.w) >= from);
}
// The smallest value of the logits' type at and above a key's: entries that reach one reach the other.
template <typename TIn>
__device__ __forceinline__ float threshold(int key) {
  const float z = key_value(key);
  if (sizeof(TIn) == 4) return z;
  const uint32_t bits = __float_as_uint(z);
  return __uint_as_float(bits & 0xffffu ? ((int)bits >= 0 ? (bits & 0xffff0000u) + 0x10000u : bits & 0xffff0000u) : bits);
}
template <typename TIn>
__device__ __forceinline__ float piece_entry(const uint4& v, int e) {
  if (sizeof(TIn) == 4) return __uint_as_float(e & 2 ? (e & 1 ? v.w : v.z) : (e & 1 ? v.y : v.x));
  const uint32_t w = e & 4 ? (e & 2 ? v.w : v.z) : (e & 2 ? v.y : v.x);
  return e & 1 ? bf16hi(w) : bf16lo(w);
}

// Where more entries of the opened units reach tau than can be ranked: a key that K and no more than can be ranked reach,
// by search between tau and the largest, two thresholds a step, into sh.low[0], and their number into sh.n_cand.  Where no
// value parts them the K-th largest, which more reach.
// (128 alternatives of 20 480 rows of 4 096 entries 6.3 ms by halves, entry by entry, down to exactly K, so 0.9 ms; a step
// waits for L2.)
template <typename TIn, int TH>
__device__ __noinline__ void refine_tau(const Slice<TIn> s, int K, float M, int tau, int n_open, int room, int32_t* status) {
  ScoreShared<TH>& sh = score_shared<TH>();
  const Units un = units_of<TH>(room);
  int flip = 0;
  __syncthreads();
  int64_t lo = tau == kNone ? order_key(-INFINITY) : tau, hi = (int64_t)order_key(M) + 1;   // fewer than K reach hi
  int c = kCand + 1;   // entries that reach lo
  while (hi - lo != 1 && c > kCand) {
    const int64_t third = hi - lo > 3 ? (hi - lo) / 3 : 1, m1 = lo + third, m2 = hi - third > m1 ? hi - third : m1;
    const float a = threshold<TIn>((int)m1), b = threshold<TIn>((int)m2);
    int va = s.edge >= 0 && s.edge_z >= a, vb = s.edge >= 0 && s.edge_z >= b;
    for_opened<TIn, TH>(s, un.open, n_open, status, [&](const uint4& v, int) {
      va += count_piece(v, a, static_cast<TIn*>(nullptr));
      vb += count_piece(v, b, static_cast<TIn*>(nullptr));
    });
    const int2 v = block_count<TH>(va, vb, sh.count, flip);
    if (v.y >= K) {
      lo = m2;
      c = v.y;
    } else if (v.x >= K) {
      lo = m1;
      c = v.x;
      hi = m2;
    } else {
      hi = m1;
    }
  }
  if (threadIdx.x == 0) {
    sh.low[0] = (int)lo;
    sh.n_cand = c;
  }
  __syncthreads();
}

// The entries of the opened units that belong to the list, where more reach tau than can be ranked: those of a refined
// tau or, where more have the K-th largest value than can be ranked, those of that value up to an index found by
// bisection.  Returns the mass of the others in the opened units.
template <typename TIn, int TH>
__device__ __noinline__ Mass select_exactly(const Slice<TIn> s, int K, float M, int tau, int n_open, int room,
                                            int32_t* status) {
  ScoreShared<TH>& sh = score_shared<TH>();
  const Units un = units_of<TH>(room);
  constexpr int N = Elem<TIn>::N;
  refine_tau<TIn, TH>(s, K, M, tau, n_open, room, status);
  tau = sh.low[0];
  const bool parted = sh.n_cand <= kCand;
  int flip = 0;
  auto walk = [&](auto f) {
    for_opened<TIn, TH>(s, un.open, n_open, status, [&](const uint4& v, int k0) {
#pragma unroll 1
      for (int e = 0; e < N; ++e) f(piece_entry<TIn>(v, e), k0 + e);
    });
    if (s.edge >= 0) f(s.edge_z, s.edge);
  };
  const float equal = key_value(tau), above = parted ? equal : key_value(tau + 1);   // (at most +infinity)
  int ilo = -1, ihi = s.entry0 + s.np * N + N;   // up to ilo: too few
  while (!parted && ihi - ilo > 1) {
    const int mid = ilo + (ihi - ilo) / 2;
    int v = 0;
    walk([&](float z, int k) { v += (z >= above || (z >= equal && k <= mid)) ? 1 : 0; });
    if (block_count<TH>(v, 0, sh.count, flip).x >= K) ihi = mid; else ilo = mid;
  }
  __syncthreads();   // (all have read the number)
  if (threadIdx.x == 0) sh.n_cand = 0;
  __syncthreads();
  Mass below = {kLowest, 0.f};
  walk([&](float z, int k) {
    if (z >= above || (z >= equal && k <= ihi)) {
      const int i = atomicAdd(&sh.n_cand, 1);
      if (ADWIN_CHK(i < kCand, status)) {
        sh.cand[i] = rank_key(z, k);
        sh.rank[i] = 0;
      }
    } else {
      below.add(z);
    }
  });
  __syncthreads();
  return below;
}

// The K largest entries of the slice into sh.sorted_z / sorted_id (fewer if it has fewer); returns their number and the
// mass of all the others in sh.rest.
template <typename TIn, int TH>
__device__ __noinline__ int select_top(const Slice<TIn> s, int K, float M, int slots, int room, int32_t* status) {
  ScoreShared<TH>& sh = score_shared<TH>();
  const Units un = units_of<TH>(room);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int flip = 0;
  // a thread reads back its own units only
  int kmin = 0x7fffffff, kmax = kNone, mine = 0;
  for (int j = 0; j < slots; ++j) {
    const int k = un.key[j * TH + tid];
    if (k == kNone) continue;
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
  const int units = block_count<TH>(mine, 0, sh.count, flip).x;
  kmin = __reduce_min_sync(0xffffffffu, lane < TH / 32 ? sh.low[lane] : 0x7fffffff);
  kmax = __reduce_max_sync(0xffffffffu, lane < TH / 32 ? sh.high[lane] : kNone);
  // tau: at least K units reach it, few more where the maxima differ.  Three thresholds a step.
  int tau = kNone;
  if (units > K) {
    int64_t lo = kmin, hi = (int64_t)kmax + 1;
    int c = units;
    const int enough = K + K / 4 + 4;
    while (hi - lo != 1 && c > enough) {
      const int64_t q = (hi - lo) >> 2, m2 = lo + ((hi - lo) >> 1), m1 = lo + (q > 0 ? q : 1), m3 = m2 + q;
      int v1 = 0, v2 = 0, v3 = 0;
      for (int j = 0; j < slots; ++j) {
        const int k = un.key[j * TH + tid];
        v1 += k >= m1 ? 1 : 0;
        v2 += k >= m2 ? 1 : 0;
        v3 += k >= m3 ? 1 : 0;
      }
      const int2 n = block_count<TH>(v1 | (v2 << 16), v3, sh.count, flip);   // (at most kSlots TH each)
      const int n1 = n.x & 0xffff, n2 = (int)((uint32_t)n.x >> 16), n3 = n.y;
      if (n3 >= K) { lo = m3; c = n3; }
      else if (n2 >= K) { lo = m2; c = n2; hi = m3 > m2 ? m3 : hi; }
      else if (n1 >= K) { lo = m1; c = n1; hi = m2 > m1 ? m2 : hi; }
      else hi = m1;
    }
    tau = (int)lo;
  }
  // the opened units, in an order of their own; the others' sums
  Mass others = {kLowest, 0.f};
  int n_mine = 0;
  for (int j = 0; j < slots; ++j) {
    const int k = un.key[j * TH + tid];
    if (k == kNone) continue;
    if (k >= tau) ++n_mine;
    else others.add(fmaxf(key_value(k), kLowest), un.sum[j * TH + tid]);
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
  const int per_warp = lane < TH / 32 ? sh.low[lane] : 0;
  const int n_open = __reduce_add_sync(0xffffffffu, per_warp);
  int at = __reduce_add_sync(0xffffffffu, lane < warp ? per_warp : 0) + before - n_mine;
  for (int j = 0; j < slots; ++j) {
    const int k = un.key[j * TH + tid];
    if (k != kNone && k >= tau) un.open[at++] = (uint16_t)(j * TH + tid);
  }
  __syncthreads();

  auto candidate = [&](float z, int k) {
    const int i = atomicAdd(&sh.n_cand, 1);
    if (i < kCand) {
      sh.cand[i] = rank_key(z, k);
      sh.rank[i] = 0;
    }
  };
  if (tau == kNone && s.np > kCand / Elem<TIn>::N) {   // every entry reaches it, more than can be ranked
    refine_tau<TIn, TH>(s, K, M, tau, n_open, room, status);
    tau = sh.low[0];
    __syncthreads();
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
  }
  const float tau_z = tau == kNone ? -INFINITY : threshold<TIn>(tau);
  // Entries below tau in the opened units: against the smallest of the units' maxima, where that is near enough
  // (an entry of the slice that is below tau too, so what vanishes beside it is nothing to the mass outside)
  Mass below = {kLowest, 0.f};
  const float ref = key_value(kmin);
  const bool near = kmin < tau && ref >= tau_z - 60.f;
  f2_t S = 0ull;
  const f2_t neg_ref = splat2(-ref);
  for_opened<TIn, TH>(s, un.open, n_open, status, [&](uint4 v, int k0) {
    const uint4 all = v;
    uint32_t in = split_piece(v, tau_z, static_cast<TIn*>(nullptr));
    while (in) {
      const int e = __ffs((int)in) - 1;
      in &= in - 1;
      candidate(piece_entry<TIn>(all, e), k0 + e);
    }
    f2_t z[Pairs<TIn>::NP];
    Pairs<TIn>::make(v, z);
    if (near) {
#pragma unroll
      for (int j = 0; j < Pairs<TIn>::NP; ++j) S = add2(S, ex2_2(mul2(add2(z[j], neg_ref), splat2(kLog2e))));
    } else {
#pragma unroll
      for (int j = 0; j < Pairs<TIn>::NP; ++j) {
        float a, b;
        upk2(z[j], a, b);
        below.add(a);
        below.add(b);
      }
    }
  });
  if (near) below = Mass{ref, hsum2(S)};
  if (s.edge >= 0) {
    if (s.edge_z >= tau_z) candidate(s.edge_z, s.edge);
    else below.add(s.edge_z);
  }
  __syncthreads();
  int n = sh.n_cand;
  if (n > kCand) {
    below = select_exactly<TIn, TH>(s, K, M, tau, n_open, room, status);
    __syncthreads();
    n = min(sh.n_cand, kCand);
  }
  // ranks: the candidates against one another, shared out over all threads
  const int wide = (n + 31) & ~31, parts = wide <= TH ? TH / wide : 1;
  if (parts > 1) {
    const int i = tid % wide, part = tid / wide;
    if (i < n && part < parts) {
      const unsigned long long key = sh.cand[i];
      int rank = 0;
      for (int j = part; j < n; j += parts) rank += sh.cand[j] > key ? 1 : 0;
      atomicAdd(&sh.rank[i], rank);
    }
    __syncthreads();
    if (tid < n) {
      const unsigned long long key = sh.cand[tid];
      sh.sorted_z[sh.rank[tid]] = rank_logit(key);
      sh.sorted_id[sh.rank[tid]] = rank_id(key);
    }
  } else {
    for (int i = tid; i < n; i += TH) {
      const unsigned long long key = sh.cand[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sh.cand[j] > key ? 1 : 0;
      sh.sorted_z[rank] = rank_logit(key);
      sh.sorted_id[rank] = rank_id(key);
    }
  }
  __syncthreads();
  for (int i = K + tid; i < n; i += TH) below.add(sh.sorted_z[i]);
  below.add(others.m, others.s);
  const Mass rest = block_mass<TH>(below, sh.red[0], sh.red[1]);
  if (tid == 0) sh.rest = rest;
  __syncthreads();
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
  ScoreShared<TH>& sh = score_shared<TH>();
  const Units un = units_of<TH>(TOP ? p.units : 0);
  SliceResult* slices = reinterpret_cast<SliceResult*>(
      score_smem + units_offset<TH>() + (TOP ? ((size_t)p.units * Units::kBytes + 15) / 16 * 16 : 0));
  constexpr int N = Elem<TIn>::N;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = (int)cluster_size(), me = C > 1 ? (int)cluster_rank() : 0;
  const int K = TOP ? p.K : 0;

  sh.list.build(p.range, p.status);
  for_rows_outside(p.range, sh.list, [&](int64_t r) {
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
    const int pieces = (int)rp.pieces, per = C == 1 ? pieces : (int)((uint32_t)(pieces + C - 1) / (uint32_t)C);
    const int first = per * me < pieces ? per * me : pieces;
    s.np = first + per < pieces ? per : pieces - first;
    s.entry0 = rp.head + first * N;
    s.src = reinterpret_cast<const uint4*>(s.row + (size_t)s.entry0 * sizeof(TIn));
    s.edge = -1;
    if (me == 0 && tid < rp.head) s.edge = tid;
    if (me == C - 1 && tid >= 32 && tid - 32 < rp.tail) s.edge = (int)p.V - rp.tail + (tid - 32);
    s.edge_z = s.edge >= 0 ? Elem<TIn>::load1(s.row, s.edge) : 0.f;
    const int trips = (s.np + kUnroll * TH - 1) / (kUnroll * TH);
    s.groups = p.groups;   // (of the longest slice: a row with a piece less must not take more room than that)
    const int slots = s.groups == 1 ? trips : (trips + s.groups - 1) / s.groups;
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
    int i = tid;
    for (int slot = 0; slot < slots; ++slot) {
      ExpSum unit;
      unit.reset();
      int key = kNone;
      for (int g = 0; g < s.groups; ++g, i += kUnroll * TH) {
        if (i - tid >= s.np) break;
        uint4 v[kUnroll];
        if (i - tid + kUnroll * TH <= s.np) {
#pragma unroll
          for (int k = 0; k < kUnroll; ++k)
            if (ADWIN_CHK(s.entry0 + (int64_t)(i + k * TH + 1) * N <= p.V, p.status)) v[k] = __ldcs(s.src + i + k * TH);
        } else {
          constexpr uint32_t kMasked = sizeof(TIn) == 2 ? 0xff80ff80u : 0xff800000u;   // -infinity
#pragma unroll
          for (int k = 0; k < kUnroll; ++k) {
            v[k] = make_uint4(kMasked, kMasked, kMasked, kMasked);
            if (i + k * TH < s.np && ADWIN_CHK(s.entry0 + (int64_t)(i + k * TH + 1) * N <= p.V, p.status))
              v[k] = __ldcs(s.src + i + k * TH);
          }
        }
        const float gm = group_max(v, static_cast<TIn*>(nullptr));
        if (TOP && i < s.np) key = max(key, order_key(gm));
        unit.merge(group_sum<TIn, kUnroll>(v, gm));
      }
      if (TOP && ADWIN_CHK(slot * TH + tid < p.units, p.status)) {
        un.key[slot * TH + tid] = key;
        un.sum[slot * TH + tid] = unit.s;
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
      const bool there = lane < TH / 32;
      const float lm = there ? sh.red[0][lane] : kLowest, ls = there ? sh.red[1][lane] : 0.f;
      const float la = there ? sh.red[2][lane] : 0.f;
      tot.m = warp_max(lm);
      const float tq = max_nan((lm - tot.m) * kLog2e, kNil), wq = ex2f(tq);
      tot.s = lane_sum(wq * ls);
      tot.a = lane_sum(wq * fmaf(ls, tq, la));
    }
    // (a slice of masked entries only is no reason to stop, a NaN or +infinity is)
    const bool sound = isfinite(tot.s) && isfinite(tot.m);
    Mass rest = {kLowest, 0.f};
    int n_top = 0;
    if (TOP && sound && (C > 1 || tot.s > 0.f)) {
      n_top = select_top<TIn, TH>(s, K, tot.m, slots, p.units, p.status);
      rest = sh.rest;
    }

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
        const bool there = lane < C;
        const float lm = there ? slices[lane].m : kLowest, ls = there ? slices[lane].s : 0.f;
        const float la = there ? slices[lane].a : 0.f;
        tot.m = warp_max(lm);
        const float tq = max_nan((lm - tot.m) * kLog2e, kNil), wq = ex2f(tq);
        tot.s = lane_sum(wq * ls);
        tot.a = lane_sum(wq * fmaf(ls, tq, la));
        Mass lr = {kLowest, 0.f};
        if (there) lr = slices[lane].rest;
        rest.m = warp_max(lr.m);
        rest.s = lane_sum(ex2f(max_nan((lr.m - rest.m) * kLog2e, kNil)) * lr.s);
        if constexpr (TOP) {
          // rank of an entry: its place in its own list and, by bisection, in the others'; equal
          // entries of an earlier slice come first, they have the lower index
          Mass losers = {kLowest, 0.f};
          for (int i2 = tid; i2 < C * K; i2 += TH) {
            const int q = i2 / K, j = i2 % K;
            if (j >= slices[q].n) continue;
            const float z = slices[q].z[j];
            // (all searches at once: a step in each list, the first one whose entries come later)
            int lo[kMaxClusterX], len[kMaxClusterX];
#pragma unroll
            for (int o = 0; o < kMaxClusterX; ++o) {
              lo[o] = 0;
              len[o] = o < C && o != q ? slices[o].n : 0;
            }
            for (int width = ADWIN_TOP_MAX; width > 0; width >>= 1) {
#pragma unroll
              for (int o = 0; o < kMaxClusterX; ++o) {
                const int at = lo[o] + width;
                if (at > len[o]) continue;
                const float x = slices[o].z[at - 1];
                if (x > z || (x == z && o < q)) lo[o] = at;
              }
            }
            int rank = j;
#pragma unroll
            for (int o = 0; o < kMaxClusterX; ++o) rank += lo[o];
            if (rank < K) {
              sh.sorted_z[rank] = z;
              sh.sorted_id[rank] = slices[q].id[j];
            } else {
              losers.add(z);
            }
          }
          losers = block_mass<TH>(losers, sh.red[0], sh.red[1]);   // (its barriers publish the list)
          rest.add(losers.m, losers.s);
        }
      }
    }
    if (me == 0) {
      const float ln_s = logf(tot.s), lse = tot.m + ln_s;
      const bool finite = isfinite(lse);
      const float nan = __int_as_float(0x7fc00000);
      if constexpr (TOP) {
        for (int j = tid; j < K; j += TH) {
          p.top_ids[r * K + j] = finite ? sh.sorted_id[j] : -1;
          p.top_logprobs[r * K + j] = finite ? (sh.sorted_z[j] - tot.m) - ln_s : nan;
        }
      }
      float listed = 1.f;   // the list's share, where it is less than half
      if (TOP && tid < 32 && finite) {
        float w = 0.f;
        for (int j = tid; j < K; j += 32) w += ex2f((sh.sorted_z[j] - tot.m) * kLog2e);
        listed = lane_sum(w) / tot.s;
      }
      if (tid == 0) {
        p.logprob[r] = (y_valid && finite) ? (zy - tot.m) - ln_s : nan;
        if (p.entropy) p.entropy[r] = finite ? fmaf(-tot.a / tot.s, kLn2, ln_s) : nan;
        if (p.lse) p.lse[r] = lse;
        if (TOP && p.rest)
          // (beside a list of less than half the mass was summed for nothing: its share is known only with the list)
          p.rest[r] = !finite ? nan : listed < 0.5f ? log1pf(-listed) : (rest.m - tot.m) + (logf(rest.s) - ln_s);
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

constexpr int kBwdUnroll = 4;

template <typename TIn, typename TOut, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) token_scores_bwd_kernel(const ScoreBwdParams p) {
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
    for (int j = tid; j <= p.K; j += TH) {
      int32_t id = -1;
      float w = 0.f;
      if (j < p.K) {
        id = p.top_ids[r * p.K + j];
        w = p.d_top[r * p.K + j];
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
      own_id[j] = id;
      own_w[j] = w;
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
    // this thread's single entries, read before the gradient may overwrite them (grad may be the logits)
    constexpr int kMine = (ADWIN_TOP_MAX + TH) / TH;
    int64_t mine[kMine];
    float z_mine[kMine];
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      mine[k] = tid + k * TH <= p.K ? own_id[tid + k * TH] : -1;
      if (mine[k] < begin || mine[k] >= end) mine[k] = -1;
      z_mine[k] = mine[k] >= 0 ? Elem<TIn>::load1(row, mine[k]) : 0.f;
    }
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
    for (int64_t i = tid; i < np; i += kBwdUnroll * TH) {
      uint4 v[kBwdUnroll];
#pragma unroll
      for (int k = 0; k < kBwdUnroll; ++k)
        if (!zero && i + k * TH < np &&
            ADWIN_CHK(entry0 + (i + k * TH + 1) * N <= p.V, p.status))
          v[k] = __ldcs(src + i + k * TH);
#pragma unroll
      for (int k = 0; k < kBwdUnroll; ++k) {
        const int64_t q = i + k * TH;
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
        } else {   // an entry at a time (2 300 bf16 rows of 50 257, fp32 gradient: 150 us, 106 at the copy rate)
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
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      if (mine[k] < 0) continue;
      float g = grad1(z_mine[k]);
      for (int j = 0; j <= p.K; ++j) g += own_id[j] == (int32_t)mine[k] ? own_w[j] : 0.f;
      if (ADWIN_CHK(mine[k] < p.V, p.status)) Elem<TOut>::store1(out, mine[k], g);
    }
    __syncthreads();
  }
  if (p.zero_tail) zero_rows_outside<TOut>(p.range, p.grad, p.ld_grad, p.V);
}

template <typename TIn, int TH, bool TOP>
cudaError_t launch_scores(ScoreParams p, int64_t clusters, int C, cudaStream_t s) {
  auto room = [](size_t units, int slices) {
    return units_offset<TH>() + (units * Units::kBytes + 15) / 16 * 16 + slices * sizeof(SliceResult);
  };
  // what the longest slice needs: its pieces (the first and the last of a row may be partial) in kSlots units to a thread at most
  const int64_t pieces = (p.V / Elem<TIn>::N + C - 1) / C, trips = (pieces + kUnroll * TH - 1) / (kUnroll * TH);
  const int64_t groups = trips <= kSlots ? 1 : (trips + kSlots - 1) / kSlots;
  p.units = TOP ? (int)((trips + groups - 1) / groups) * TH : 0;
  p.groups = (int)groups;
  const size_t smem = room(p.units, C > 1 ? C : 0);
  // (one limit for every launch of this kernel: launches of other threads may come in between)
  constexpr size_t limit = units_offset<TH>() + kSlots * TH * Units::kBytes + kMaxClusterX * sizeof(SliceResult);
  const cudaError_t e = shared_limit<token_scores_kernel<TIn, TH, TOP>>(limit);
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
  // Few rows: clusters of two to eight CTAs with 512 threads share a row, as many as half of the SMs leave each.
  // Many: a CTA of 128 threads each, eight per SM.  Calls between about 75 and 600 rows are the weak side of this rule:
  // 75 rows keep half of the SMs idle.  151 936 bf16 entries, us without alternatives / with 20, read once at the
  // copy rate in brackets: 8 rows 5.6 / 12.5 (0.4), 37 (four CTAs to a row) 14.7 / 30.2 (1.7), 38 (two) 10.4 / 17.5, 74 11.3 / 18.6 (3.4), 75 23.9 / 34.5 (3.5),
  // 148 24.7 / 35.6 (6.9), 300 30.7 / 43.6 (13.9), 600 48.7 / 65.2 (27.8), 2 400 125 / 169 (111); fp32 74 12.8 / 20.7, 75
  // 35.9 / 51.7, 600 62.4 / 82.2 (55.6), 2 400 227 / 286 (222).
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
  while (rows * splits * 2 <= room && pieces >= splits * 4 * kBwdUnroll * 256) splits *= 2;
  p.splits = (int)splits;
  int64_t grid = (int64_t)sm_count * 32;
  if (grid > rows * splits) grid = rows * splits;
  // 128 threads to a row of fewer than 8 000 pieces: what a row costs outside its sweep is hidden by twice as many rows
  // per SM (20 480 bf16 rows of 8 192 178 -> 138 us, of 16 384 269 -> 233, 10 240 of 50 000 346.5 -> 344). 256 to longer
  // ones (5 120 of 100 000 344 -> 337 us, of 151 936 510 -> 492) and where four per SM take every row (320 of 8 192
  // 8.1 -> 7.5 us)
  const bool narrow = pieces < 8000 && rows > (int64_t)sm_count * 4;
#define ADWIN_BWD(TIN, TOUT)                                                                                    \
  (narrow ? launch_chained(token_scores_bwd_kernel<TIN, TOUT, 128>, (unsigned)grid, 128, 0, 1, s, p)            \
          : launch_chained(token_scores_bwd_kernel<TIN, TOUT, 256>, (unsigned)grid, 256, 0, 1, s, p))
  if (bf) return grad_dtype == ADWIN_BF16 ? ADWIN_BWD(__nv_bfloat16, __nv_bfloat16) : ADWIN_BWD(__nv_bfloat16, float);
  return grad_dtype == ADWIN_BF16 ? ADWIN_BWD(float, __nv_bfloat16) : ADWIN_BWD(float, float);
#undef ADWIN_BWD
}

}  // namespace adwin
