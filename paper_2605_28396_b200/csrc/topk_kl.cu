// Divergence of the student from a teacher known by its K most likely alternatives and the mass
// outside them, with the gradient: one read of the student's logits, one write of the gradient.
//
// Categories c: the alternatives j = 1..K, each an entry id_j of the vocabulary, and the rest r,
//   P_j = exp(z_id_j - lse),   P_r = sum over all other entries of p_k,   Q_j, Q_r the teacher's:
//   reverse  KL = sum_c P_c (log P_c - log Q_c),    g_k = alpha p_k (D_c(k) - KL),   D_c = log P_c - log Q_c
//   forward  KL = sum_c Q_c (log Q_c - log P_c),    g_k = alpha (p_k - Q_c(k) p_k / P_c(k)).
// So every entry of the rest gets p_k times one coefficient of the row.  P_r is summed over the entries
// of the rest alone (1 - sum_j P_j would have no correct digit where the list holds nearly everything;
// where it holds less than half, log P_r is better made of it: log P_r = -0.02 is under 5e-7 of itself off in place of 3e-6):
// a thread masks the listed entries out of the pieces they lie in, which it finds in a chain in shared
// memory, empty for most threads.  |g|^2 needs sum p_k^2 over the rest beside it.
//
// A row is read from memory once: its second read comes while it is still in L2 (the first asks for it to be
// kept, the second and the gradient's stores to go first; a CTA, or a cluster with a slice of the
// row each, has one row at a time).  Several CTAs per SM fill one another's gaps between the sweeps.  The warps meet
// twice a row: when their sums are there, and when one more warp has made the row's scalars of
// them.  In a cluster that warp alone exchanges the CTAs' sums: a cluster barrier would have every
// thread wait for its gradient's stores.  It
// also looks the rows up, sums the few entries beside the 16-byte pieces and writes the outputs;
// another prepares the lists, in three steps a row apart (index, logit, chains and sums), so that
// it never waits for its loads.
#include <atomic>

#include "adwin_common.cuh"
#include "adwin_internal.h"
#include "exp_sums.cuh"
#include "row_list.cuh"
#include "tc_pipeline.cuh"

namespace adwin {
namespace {

constexpr int kGroup = 4;        // pieces a thread takes at a time
constexpr int kMaxCtas = 8;      // of a cluster
constexpr int kInfos = 8;        // rows that are known at a time
constexpr int kPerLane = ADWIN_TOP_MAX / 32;
constexpr int kChains = 128;

struct TopkParams {
  const void* logits;
  int64_t V, ld;
  RowRange range;            // processed positions
  const int32_t* window;     // positions with gradient, within them (null: T)
  const int32_t* rollout;
  const int32_t* tokens;
  const int32_t* top_ids;
  const float *top_logprobs, *rest;   // rest: may be null
  int K;
  float alpha;
  bool forward, zero_tail;
  void* grad;                // may be null
  int64_t ld_grad;
  float *kl, *logratio, *gsq, *lse;   // gsq, lse: may be null
  int32_t* status;
  uint64_t limit_ns;         // of the wait for the records
};

// What the threads have to know of a row.
struct RowInfo {
  const char* row;       // its logits, or null: no more rows
  char* out;             // its gradient, or null
  int64_t r;
  int entry0;            // vocabulary index of the slice's first piece
  int np;                // pieces of the slice
  int head, tail;        // entries beside the row's pieces that belong to this CTA
  int y;
};

// The listed entries of a row, in chains by the thread whose pieces hold them; an index that comes
// twice is found in its chain.
struct TopList {
  int32_t id[ADWIN_TOP_MAX];      // -1: none
  float z[ADWIN_TOP_MAX], lq[ADWIN_TOP_MAX];
  int32_t slot[ADWIN_TOP_MAX];    // where it lies among its thread's pieces, or -1: not in this CTA's
  int16_t owner[ADWIN_TOP_MAX];   // its thread
  int16_t next[ADWIN_TOP_MAX];
  int32_t counts[ADWIN_TOP_MAX];  // 0: none, or an index that the list has already
  int32_t first[kChains];         // -1: an empty chain
  float lq_rest;
  // Sums over the list, e_j = exp(z_j - zmax):  s = sum e_j;  and with x_j = (z_j - zmax) - lq_j
  // a = sum e_j x_j (reverse) or sum Q_j x_j (forward), q = sum Q_j
  float zmax, s, a, q;
};

struct alignas(16) SumRecord {   // (written to a cluster's other CTAs in one piece)
  float m, s, q;   // reference, sum e, sum e^2 over entries of the rest
  float pad;
};

// Scalars of a row.
struct TopScalars {
  float M, ln_s, inv_s;   // reference, log and inverse of the whole sum against it
  float kl, d_rest;
  // g_k = alpha c_rest exp(z_k - m_rest) for entries of the rest: against their own largest, for
  // the forward divergence divides by their mass, however far that is below the listed entries'
  float m_rest, c_rest;
  float gsq_rest;         // sum (g_k / alpha)^2 over them
};

template <int TH>
struct TopkShared {
  static constexpr int kWarps = TH / 32 + 1;
  RowList list;
  RowInfo info[kInfos];
  TopList lists[3];
  TopScalars scalars;
  SumRecord rec[2][kWarps];          // of the CTA's warps
  SumRecord slice[2][kMaxCtas];      // of the cluster's CTAs
  unsigned long long complete[2];    // mbarriers: so they are there
  int abort;
};
static_assert(alignof(TopkShared<128>) == 16 && sizeof(SumRecord) == 16, "records are stored 16 bytes at a time");

// A row's first read and its second.
__device__ __forceinline__ uint64_t keep_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t drop_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 read16(const uint4* src, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(src), "l"(policy));
  return v;
}
// A logit as it lies in memory, so that a register can wait for it.
__device__ __forceinline__ uint32_t raw_logit(const void* row, int i, float*) {
  return __ldg(static_cast<const uint32_t*>(row) + i);
}
__device__ __forceinline__ uint32_t raw_logit(const void* row, int i, __nv_bfloat16*) {
  return __ldg(static_cast<const uint16_t*>(row) + i);
}
__device__ __forceinline__ float logit_of(uint32_t raw, float*) { return __uint_as_float(raw); }
__device__ __forceinline__ float logit_of(uint32_t raw, __nv_bfloat16*) { return bf16lo(raw); }

template <typename TIn>
__device__ __forceinline__ uint4 masked_piece() {
  constexpr uint32_t w = sizeof(TIn) == 2 ? 0xff80ff80u : 0xff800000u;   // -infinity
  return make_uint4(w, w, w, w);
}
// Entry `e` of a group of pieces becomes -infinity.
template <typename TIn, int U>
__device__ __forceinline__ void mask_entry(uint4 (&v)[U], int e) {
  const int word = sizeof(TIn) == 4 ? e : e >> 1;
  const uint32_t keep = sizeof(TIn) == 4 ? 0u : (e & 1 ? 0xffffu : 0xffff0000u);
  const uint32_t put = sizeof(TIn) == 4 || (e & 1) ? 0xff800000u : 0xff80u;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (word == 4 * k) v[k].x = (v[k].x & keep) | put;
    if (word == 4 * k + 1) v[k].y = (v[k].y & keep) | put;
    if (word == 4 * k + 2) v[k].z = (v[k].z & keep) | put;
    if (word == 4 * k + 3) v[k].w = (v[k].w & keep) | put;
  }
}

// Sums over entries of the rest, of one thread.
struct RestSum {
  float m;
  f2_t S, Q;
  __device__ __forceinline__ void reset() {
    m = kLowest;
    S = Q = 0ull;
  }
  __device__ __forceinline__ void raise(float x) {
    if (x > m) {
      const f2_t f = splat2(exp_below(m, x));
      S = mul2(S, f);
      Q = mul2(Q, mul2(f, f));
      m = x;
    }
  }
  __device__ __forceinline__ void add(f2_t z, f2_t neg_m) {
    const f2_t e = ex2_2(mul2(add2(z, neg_m), splat2(kLog2e)));
    S = add2(S, e);
    Q = fma2(e, e, Q);
  }
};

// Gradient at a listed entry, before alpha.
__device__ __forceinline__ float listed_grad(const TopScalars& t, float z, float lq, bool forward) {
  const float p = exp_below(z, t.M) * t.inv_s;
  if (forward) return p - expf(lq);
  return p == 0.f ? 0.f : p * ((((z - t.M) - t.ln_s) - lq) - t.kl);
}

template <typename TIn, typename TOut, int TH>
struct TopkCta {
  static constexpr int N = Elem<TIn>::N, NP = Pairs<TIn>::NP;
  static constexpr int kWarps = TH / 32 + 1;   // those that sum
  const TopkParams& p;
  TopkShared<TH>& sh;
  const int C, me, tid, lane, warp;

  __device__ __forceinline__ void publish(int par, float m, float s, float q) const {
    if (lane == 0) sh.rec[par][warp] = SumRecord{m, s, q, 0.f};
  }
  // Sum of n records, in every lane (n <= 32).
  __device__ __forceinline__ SumRecord sum_of(const SumRecord* r, int n) const {
    SumRecord x = {kLowest, 0.f, 0.f, 0.f};
    if (lane < n) x = r[lane];
    const float m = warp_max(x.m), w = exp_below(x.m, m);
    float s = w * x.s, q = w * w * x.q;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      q += __shfl_xor_sync(0xffffffffu, q, o);
    }
    return SumRecord{m, s, q, 0.f};
  }
  // The row's warp: the sum over the row, or false: the other CTAs' did not come in time.  A record's
  // place is free: its last content, two rows ago, was read before any CTA sent what this one needed to come here.
  __device__ __forceinline__ bool row_sum(int i, SumRecord& x) const {
    const int par = i & 1;
    x = sum_of(sh.rec[par], kWarps);
    if (C == 1) return true;
    const uint32_t bar = smem_u32(&sh.complete[par]);
    if (lane < C) {
      remote_store4(map_to_rank(smem_u32(&sh.slice[par][me]), (uint32_t)lane), x.m, x.s, x.q, 0.f);
      tc::bar_arrive_cluster(map_to_rank(bar, (uint32_t)lane));
    }
    const bool ok = __all_sync(0xffffffffu, wait_cluster(bar, (i >> 1) & 1));
    if (ok) x = sum_of(sh.slice[par], C);
    return ok;
  }
  // Waits for a phase of a barrier that the cluster's CTAs arrive on, and sees what they wrote before.
  __device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity) const {
    const uint64_t t0 = tc::timer_ns();
    for (;;) {
#pragma unroll 1
      for (int k = 0; k < 64; ++k) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if (p.limit_ns < 16) return false;   // (diagnostic: what is not there right now has run out)
      }
      if (tc::timer_ns() - t0 > p.limit_ns) return false;
    }
  }
  __device__ __forceinline__ const RowInfo& info_of(int o) const { return sh.info[o % kInfos]; }

  // ------------------------------------------------------------------ the row's warp
  struct Cursor {
    int64_t n, rows, step;
    int b;                     // sequence of the list that holds row n, or one before it
  };
  __device__ __forceinline__ void look_up(int o, Cursor& c) const {
    int64_t r = -1;
    if (p.range.listed()) {
      if (c.n < c.rows) {
        while (sh.list.off[c.b + 1] <= (int)c.n) ++c.b;
        r = (int64_t)c.b * p.range.T + ((int)c.n - sh.list.off[c.b]);
        c.n += c.step;
      }
    } else {
      while (c.n < c.rows && r < 0) {
        r = sh.list.row(p.range, c.n);
        c.n += c.step;
      }
    }
    RowInfo i = {};
    i.r = r;
    if (r >= 0) {
      i.row = static_cast<const char*>(p.logits) + (size_t)r * p.ld * sizeof(TIn);
      const RowPieces rp = RowPieces::of<TIn>(i.row, p.V);
      const int pieces = (int)rp.pieces, per = (int)((uint32_t)(pieces + C - 1) / (uint32_t)C);
      const int first = per * me < pieces ? per * me : pieces;
      i.np = first + per < pieces ? per : pieces - first;
      i.entry0 = rp.head + first * N;
      i.head = me == 0 ? rp.head : 0;
      i.tail = me == C - 1 ? rp.tail : 0;
      i.y = __ldg(p.tokens + r);
      if (p.grad) {
        bool inside = true;
        if (!p.range.window && p.window) {   // (otherwise every processed row has a gradient)
          const int64_t b = r / p.range.T;
          const RowRange w = {p.window, p.rollout, p.range.B, p.range.T};
          inside = r - b * p.range.T < w.end(b);
        }
        if (inside) i.out = static_cast<char*>(p.grad) + (size_t)r * p.ld_grad * sizeof(TOut);
      }
    }
    if (lane == 0) sh.info[o % kInfos] = i;
    __syncwarp();
  }

  // An entry beside the slice's pieces that this lane holds, or -1, and its logit.
  __device__ __forceinline__ int edge_of(const RowInfo& i) const {
    if (lane < i.head) return lane;
    if (lane >= 16 && lane - 16 < i.tail) return (int)p.V - i.tail + (lane - 16);
    return -1;
  }
  __device__ __forceinline__ uint32_t edge_logit(int o) const {
    const RowInfo& i = info_of(o);
    const int e = i.row ? edge_of(i) : -1;
    return e >= 0 ? raw_logit(i.row, e, static_cast<TIn*>(nullptr)) : 0u;
  }
  __device__ __forceinline__ int listed(const TopList& l, int e) const {
    int found = -1;
    if (__any_sync(0xffffffffu, e >= 0)) {
      for (int j = p.K - 1; j >= 0; --j)
        if (l.id[j] == e) found = j;          // (the first one counts)
    }
    return e >= 0 ? found : -1;
  }

  __device__ __forceinline__ TopScalars make_scalars(const SumRecord& x, const TopList& l) const {
    const float m = x.m, s = x.s, q = x.q;
    const float zmax = l.zmax, le = l.s, la = l.a, lqs = l.q, lqr = l.lq_rest;
    TopScalars t;
    const float M = fmaxf(m, zmax), wr = exp_below(m, M), wt = exp_below(zmax, M);
    const float sum = fmaf(wr, s, wt * le);
    t.M = M;
    t.ln_s = logf(sum);
    t.inv_s = 1.f / sum;
    t.m_rest = m;
    // (beside a list that holds less than half, what it leaves of 1 has no rounding of the sums' size in it)
    const float pl = wt * le * t.inv_s, pr = wr * s * t.inv_s;
    const float lpr = !(s > 0.f) ? -INFINITY : pl < 0.5f ? log1pf(-pl) : (m - M) + (logf(s) - t.ln_s);
    t.d_rest = lpr - lqr;
    const float shift = (zmax - M) - t.ln_s;   // log P_j - lq_j = x_j + shift
    float kl;
    t.c_rest = 0.f;   // (no entry is left, or none with any mass)
    if (p.forward) {
      const float qr = expf(lqr);
      kl = -(lqs == 0.f ? la : fmaf(lqs, shift, la));
      kl += qr == 0.f ? 0.f : qr * -t.d_rest;
      if (s != 0.f) t.c_rest = wr * t.inv_s - qr / s;
    } else {
      const float pt = wt * t.inv_s;
      kl = pt == 0.f || le == 0.f ? 0.f : pt * fmaf(le, shift, la);
      if (s != 0.f) {
        kl += pr == 0.f ? 0.f : pr * t.d_rest;
        t.c_rest = wr == 0.f ? 0.f : (t.d_rest - kl) * (wr * t.inv_s);
      }
    }
    if (!(sum > 0.f)) kl = t.c_rest = __int_as_float(0x7fc00000);   // nothing is left, or NaN
    t.gsq_rest = t.c_rest * t.c_rest * q;
    t.kl = kl;
    return t;
  }

  __device__ __forceinline__ void write_outputs(const RowInfo& info, const TopList& l, const TopScalars& t) const {
    const int y = info.y;
    const bool y_valid = y >= 0 && (int64_t)y < p.V;
    int jy = ADWIN_TOP_MAX;
    float gl = 0.f;
    for (int k = lane; k < p.K; k += 32) {
      if (!l.counts[k]) continue;
      if (l.id[k] == y) jy = k;
      if (p.gsq) {
        const float g = listed_grad(t, l.z[k], l.lq[k], p.forward);
        gl = fmaf(g, g, gl);
      }
    }
    jy = __reduce_min_sync(0xffffffffu, jy);
    gl = lane_sum(gl);
    if (lane == 0) {
      const float lse = t.M + t.ln_s;
      p.kl[info.r] = t.kl;
      p.logratio[info.r] = !y_valid ? __int_as_float(0x7fc00000)
                           : jy < ADWIN_TOP_MAX ? ((l.z[jy] - t.M) - t.ln_s) - l.lq[jy] : t.d_rest;
      if (p.gsq) p.gsq[info.r] = p.alpha * p.alpha * (t.gsq_rest + gl);
      if (p.lse) p.lse[info.r] = lse;
      int bits = 0;
      if (!y_valid) bits |= ADWIN_DEV_TOKEN_RANGE;
      if (!isfinite(lse) || !isfinite(t.kl)) bits |= ADWIN_DEV_NONFINITE;
      if (bits) atomicOr(p.status, bits);
    }
  }

  __device__ __forceinline__ void row_warp() {
    TIn* const type = nullptr;
    Cursor c = {(int64_t)(blockIdx.x / C), sh.list.count(p.range), (int64_t)(gridDim.x / C), 0};
    for (int o = 0; o < 4; ++o) look_up(o, c);
    __syncthreads();   // the lists may be prepared
    uint32_t z_here = edge_logit(0), z_next = edge_logit(1);
    __syncthreads();
    for (int i = 0;; ++i) {
      const RowInfo& info = info_of(i);
      if (!info.row) break;
      const TopList& l = sh.lists[i % 3];
      const int e = edge_of(info), j = listed(l, e);
      const float z = e >= 0 ? logit_of(z_here, type) : -INFINITY;
      {
        const float x = j >= 0 ? -INFINITY : z, m = fmaxf(warp_max(x), kLowest), w = exp_below(x, m);
        publish(i & 1, m, lane_sum(w), lane_sum(w * w));
      }
      look_up(i + 4, c);
      __syncthreads();   // the warps' sums are there
      SumRecord x;
      const bool there = row_sum(i, x);
      const TopScalars s = make_scalars(x, l);
      if (lane == 0) {
        sh.scalars = s;
        if (!there) sh.abort = 1;
      }
      __syncthreads();
      if (!there) break;
      const TopScalars t = sh.scalars;
      if (info.out && e >= 0)
        Elem<TOut>::store1(info.out, e, p.alpha * (j >= 0 ? listed_grad(t, z, l.lq[j], p.forward)
                                                          : t.c_rest * exp_below(z, t.m_rest)));
      if (me == 0) write_outputs(info, l, t);
      z_here = z_next;
      z_next = edge_logit(i + 2);
    }
  }

  // ------------------------------------------------------------------ the lists' warp
  // Step 1: a row's list is asked for.
  struct Asked {
    int32_t id[kPerLane];
    float lq[kPerLane], rest;
  };
  __device__ __forceinline__ void ask(int o, Asked& a) const {
    const RowInfo& i = info_of(o);
    const int64_t r = i.row ? i.r : -1;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      const int j = lane + 32 * k;
      a.id[k] = -1;
      a.lq[k] = 0.f;
      if (r >= 0 && j < p.K) {
        a.id[k] = __ldg(p.top_ids + r * p.K + j);
        a.lq[k] = __ldg(p.top_logprobs + r * p.K + j);
      }
    }
    a.rest = r >= 0 && p.rest ? __ldg(p.rest + r) : 0.f;
  }
  // Step 2: so are its logits.
  struct Gathered {
    Asked a;
    uint32_t z[kPerLane];
  };
  __device__ __forceinline__ void gather(int o, const Asked& a, Gathered& g) const {
    const char* row = info_of(o).row;
    g.a = a;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      if (g.a.id[k] < -1 || (int64_t)g.a.id[k] >= p.V) {
        if (me == 0) atomicOr(p.status, (int32_t)ADWIN_DEV_TOKEN_RANGE);
        g.a.id[k] = -1;
      }
      g.z[k] = 0u;
      if (g.a.id[k] >= 0) g.z[k] = raw_logit(row, g.a.id[k], static_cast<TIn*>(nullptr));
    }
  }
  // Step 3: its chains and sums, into lists[o % 3].
  __device__ __forceinline__ void prepare(int o, const Gathered& g) {
    TopList& l = sh.lists[o % 3];
    const RowInfo& i = info_of(o);
    for (int k = lane; k < kChains; k += 32) l.first[k] = -1;
    __syncwarp();
    int chain[kPerLane];
    float z[kPerLane];
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      const int j = lane + 32 * k;
      const int32_t id = g.a.id[k];
      z[k] = logit_of(g.z[k], static_cast<TIn*>(nullptr));
      chain[k] = id & (kChains - 1);
      if (j >= p.K) continue;
      int owner = -1, slot = -1;
      const int e = id - i.entry0;
      if (id >= 0 && e >= 0 && e < i.np * N) {
        const uint32_t piece = (uint32_t)e / N;
        owner = (int)(piece % TH);
        slot = (int)(piece / TH);
        chain[k] = owner & (kChains - 1);
      }
      l.id[j] = id;
      l.lq[j] = g.a.lq[k];
      l.z[j] = z[k];
      l.slot[j] = slot;
      l.owner[j] = (int16_t)owner;
      if (id >= 0) l.next[j] = (int16_t)atomicExch(&l.first[chain[k]], j);   // (the order of a chain does not matter)
    }
    __syncwarp();
    float zmax = kLowest;
    bool counts[kPerLane];
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      const int j = lane + 32 * k;
      const int32_t id = g.a.id[k];
      counts[k] = id >= 0;
      if (id >= 0) {      // an index that the list has already does not count
        for (int x = l.first[chain[k]]; x >= 0; x = l.next[x])
          if (x < j && l.id[x] == id) counts[k] = false;
        if (!counts[k] && me == 0) atomicOr(p.status, (int32_t)ADWIN_DEV_TOKEN_RANGE);
      }
      if (j < p.K) l.counts[j] = counts[k];
      if (counts[k]) zmax = fmaxf(zmax, z[k]);
    }
    zmax = warp_max(zmax);
    float s = 0.f, a = 0.f, q = 0.f;
    double mass = 0.0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      if (!counts[k]) continue;
      const float lq = g.a.lq[k], e = exp_below(z[k], zmax), x = (z[k] - zmax) - lq, w = p.forward ? expf(lq) : e;
      s += e;
      if (p.forward) q += w;
      a += w == 0.f ? 0.f : w * x;
      if (!p.rest) mass += exp((double)lq);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, x);
      a += __shfl_xor_sync(0xffffffffu, a, x);
      q += __shfl_xor_sync(0xffffffffu, q, x);
      if (!p.rest) mass += __shfl_xor_sync(0xffffffffu, mass, x);
    }
    const float lqr = p.rest ? g.a.rest : (float)log(fmax(1.0 - mass, 5.9604644775390625e-8));   // 2^-24
    if (lane == 0) {
      l.lq_rest = lqr;
      l.zmax = zmax;
      l.s = s;
      l.a = a;
      l.q = q;
    }
    __syncwarp();
  }
  __device__ __forceinline__ void list_warp() {
    __syncthreads();
    Asked asked;
    Gathered got;
    ask(0, asked);
    gather(0, asked, got);
    ask(1, asked);
    prepare(0, got);
    gather(1, asked, got);
    ask(2, asked);
    __syncthreads();
    for (int i = 0; info_of(i).row; ++i) {
      // beside the sums of row i: the list of the next, in a buffer that row i - 2 has left
      prepare(i + 1, got);
      gather(i + 2, asked, got);
      ask(i + 3, asked);
      __syncthreads();
      __syncthreads();
      if (*static_cast<volatile int*>(&sh.abort)) break;
    }
  }

  // ------------------------------------------------------------------ the threads that sweep
  // Which of this thread's slots (its pieces tid, tid + TH, ...) hold listed entries; with more than 32, which may.
  __device__ __forceinline__ uint32_t marks(const TopList& l) const {
    uint32_t m = 0;
    for (int k = l.first[tid & (kChains - 1)]; k >= 0; k = l.next[k])
      if (l.owner[k] == tid) m |= 1u << (l.slot[k] & 31);
    return m;
  }

  __device__ __forceinline__ void sweeps() {
    const uint64_t keep = keep_policy(), drop = drop_policy();
    __syncthreads();
    __syncthreads();
    for (int i = 0;; ++i) {
      const RowInfo& info = info_of(i);
      if (!info.row) break;
      const TopList& l = sh.lists[i % 3];
      const int entry0 = info.entry0, np = info.np;
      char* out = info.out;
      const uint4* src = reinterpret_cast<const uint4*>(info.row + (size_t)entry0 * sizeof(TIn));
      const uint32_t marked = marks(l);
      // Pieces j, j + TH, ... of this thread; those behind the slice are masked.
      auto take = [&](int j, uint64_t policy, uint4 (&v)[kGroup]) {
        if (j + (kGroup - 1) * TH < np) {
#pragma unroll
          for (int k = 0; k < kGroup; ++k)
            if (ADWIN_CHK(entry0 + (int64_t)(j + k * TH + 1) * N <= p.V, p.status)) v[k] = read16(src + j + k * TH, policy);
        } else {
#pragma unroll
          for (int k = 0; k < kGroup; ++k) {
            v[k] = masked_piece<TIn>();
            if (j + k * TH < np && ADWIN_CHK(entry0 + (int64_t)(j + k * TH + 1) * N <= p.V, p.status))
              v[k] = read16(src + j + k * TH, policy);
          }
        }
      };
      RestSum acc;
      acc.reset();
      const uint64_t first = out ? keep : drop;
#pragma unroll 1
      for (int j = tid, slot = 0; j < np; j += kGroup * TH, slot += kGroup) {
        uint4 v[kGroup];
        take(j, first, v);
        // the next group's lines on their way into L2 (5 120 rows of 151 936 bf16 entries: 720 -> 690 us)
        if ((lane & 7) == 0) {
#pragma unroll
          for (int k = 0; k < kGroup; ++k)
            if (j + (k + kGroup) * TH < np) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + j + (k + kGroup) * TH));
        }
        if (marked >> (slot & 31) & ((1u << kGroup) - 1)) {
#pragma unroll 1
          for (int x = l.first[tid & (kChains - 1)]; x >= 0; x = l.next[x]) {
            const int at = l.slot[x] - slot;
            if (l.owner[x] == tid && at >= 0 && at < kGroup) mask_entry<TIn>(v, at * N + ((l.id[x] - entry0) & (N - 1)));
          }
        }
        acc.raise(group_max(v, static_cast<TIn*>(nullptr)));
        const f2_t neg_m = splat2(-acc.m);
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          f2_t z[NP];
          Pairs<TIn>::make(v[k], z);
#pragma unroll
          for (int x = 0; x < NP; ++x) acc.add(z[x], neg_m);
        }
      }
      {
        const float m = warp_max(acc.m), w = exp_below(acc.m, m);
        float s = w * hsum2(acc.S), q = w * w * hsum2(acc.Q);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) {
          s += __shfl_xor_sync(0xffffffffu, s, x);
          q += __shfl_xor_sync(0xffffffffu, q, x);
        }
        publish(i & 1, m, s, q);
      }
      __syncthreads();     // the row's warp makes the scalars
      __syncthreads();
      if (*static_cast<volatile int*>(&sh.abort)) break;
      if (!out) continue;
      out += (size_t)entry0 * sizeof(TOut);
      constexpr int kOutPiece = N * (int)sizeof(TOut), kOutAlign = kOutPiece < 16 ? kOutPiece : 16;
      const bool wide = (reinterpret_cast<uintptr_t>(out) & (kOutAlign - 1)) == 0;
      const f2_t neg_m = splat2(-sh.scalars.m_rest), coef = splat2(p.alpha * sh.scalars.c_rest);
      auto gradient = [&](const uint4& v, f2_t (&g)[NP]) {
        f2_t z[NP];
        Pairs<TIn>::make(v, z);
#pragma unroll
        for (int x = 0; x < NP; ++x) g[x] = mul2(coef, ex2_2(mul2(add2(z[x], neg_m), splat2(kLog2e))));
      };
      if (!wide) {   // rows of the gradient off its pieces' boundaries: an entry at a time (2 300 bf16 rows of 50 257, fp32: 172 us over 106)
#pragma unroll 1
        for (int j = tid; j < np; j += TH) {
          f2_t g[NP];
          gradient(read16(src + j, drop), g);
#pragma unroll
          for (int x = 0; x < NP; ++x) {
            float a, b;
            upk2(g[x], a, b);
            Elem<TOut>::store1(out, (int64_t)j * N + 2 * x, a);
            Elem<TOut>::store1(out, (int64_t)j * N + 2 * x + 1, b);
          }
        }
      }
#pragma unroll 1
      for (int j = tid, slot = 0; j < np; j += kGroup * TH, slot += kGroup) {
        const bool any = marked >> (slot & 31) & ((1u << kGroup) - 1);
        if (wide) {
          uint4 v[kGroup];
          take(j, drop, v);
#pragma unroll
          for (int k = 0; k < kGroup; ++k) {
            if (j + k * TH >= np) break;
            f2_t g[NP];
            gradient(v[k], g);
            store_pairs<TOut>(out + (size_t)(j + k * TH) * kOutPiece, g);
          }
        }
        if (any) {   // the listed entries among them once more (a thread's stores to one place keep their order)
#pragma unroll 1
          for (int x = l.first[tid & (kChains - 1)]; x >= 0; x = l.next[x]) {
            if (l.owner[x] != tid || l.slot[x] < slot || l.slot[x] >= slot + kGroup || !l.counts[x]) continue;
            const float gl = p.alpha * listed_grad(sh.scalars, l.z[x], l.lq[x], p.forward);
            Elem<TOut>::store1(out, l.id[x] - entry0, gl);
          }
        }
      }
    }
  }
};

template <typename TIn, typename TOut, int TH, int CTAS>
__global__ void __launch_bounds__(TH + 64, CTAS) topk_kl_kernel(const TopkParams p) {
  chain();
  extern __shared__ __align__(16) uint8_t smem[];
  TopkShared<TH>& sh = *reinterpret_cast<TopkShared<TH>*>(smem);
  uint32_t nc;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(nc));
  const int C = (int)nc, me = C > 1 ? (int)cluster_rank() : 0;
  const int tid = threadIdx.x, warp = tid >> 5;

  sh.list.build(p.range, p.status);
  if (p.window && !p.range.window && blockIdx.x == 0)
    for (int64_t b = tid; b < p.range.B; b += blockDim.x)
      if (p.window[b] < 0) atomicOr(p.status, (int32_t)ADWIN_DEV_WINDOW);
  for_rows_outside(p.range, sh.list, [&](int64_t r) {
    p.kl[r] = 0.f;
    p.logratio[r] = 0.f;
    if (p.gsq) p.gsq[r] = 0.f;
    if (p.lse) p.lse[r] = 0.f;
  });
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) tc::bar_init(smem_u32(&sh.complete[i]), (uint32_t)C);
    sh.abort = 0;
    tc::bar_init_fence();
  }
  __syncthreads();
  if (C > 1) cluster_sync_all();   // every CTA and its barriers are there before anything is sent to one
  TopkCta<TIn, TOut, TH> cta = {p, sh, C, me, tid, tid & 31, warp};
  if (warp == TH / 32) cta.row_warp();
  else if (warp == TH / 32 + 1) cta.list_warp();
  else cta.sweeps();
  __syncthreads();
  if (tid == 0 && sh.abort) atomicOr(p.status, (int32_t)ADWIN_DEV_TIMEOUT);
  if (C > 1) cluster_sync_all();   // none leaves while another may still send to it
  if (p.zero_tail && p.grad) {
    const RowRange w = {p.window, p.rollout, p.range.B, p.range.T};
    zero_rows_outside<TOut>(w, p.grad, p.ld_grad, p.V);
  }
}

template <typename TIn, typename TOut, int TH, int CTAS>
cudaError_t launch_plan(const TopkParams& p, int C, int64_t rows, int sm_count, cudaStream_t s) {
  const size_t smem = sizeof(TopkShared<TH>);
  auto kernel = topk_kl_kernel<TIn, TOut, TH, CTAS>;
  cudaError_t e = shared_limit<topk_kl_kernel<TIn, TOut, TH, CTAS>>(smem);
  if (e != cudaSuccess) return e;
  // as many clusters as the GPU holds at a time: their CTAs go on from row to row
  static std::atomic<int> held[4][kKnownDevices];
  int log_c = 0;
  while ((1 << log_c) < C) ++log_c;
  int n = sm_count * CTAS;
  if (C > 1) e = per_device(held[log_c], n, [&](int& clusters) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sm_count * CTAS / C * C));
    cfg.blockDim = dim3(TH + 64);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t asked = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    return asked == cudaSuccess && clusters < 1 ? cudaErrorInvalidConfiguration : asked;
  });
  if (e != cudaSuccess) return e;
  const int64_t clusters = n < rows ? n : rows;
  return launch_chained(kernel, (unsigned)(clusters * C), TH + 64, smem, C, s, p);
}

template <typename TIn, typename TOut>
cudaError_t launch(const TopkParams& p, int64_t rows, int sm_count, cudaStream_t s) {
  const int64_t pieces = (p.V + Elem<TIn>::N - 1) / Elem<TIn>::N;
  // few rows: several CTAs to a row, as long as each has two groups of pieces to a thread
  int C = 1;
  while (C < kMaxCtas && rows * C * 2 <= sm_count && pieces >= (int64_t)C * 2 * 1024) C *= 2;
  // Many: as many threads to a row as leave each a few groups of pieces, about 32 warps per SM in all (bf16, us for 128
  // threads x 8 CTAs per SM / 256 x 4 / 512 x 2 / 960 x 1: 18 432 rows of 4 096 entries 225 / 369 / 552 / -,
  // 2 560 of 32 000 139 / 129 / 136 / -, 2 300 of 50 257 116 / 104 / 107 / -, 5 120 of 151 936 - / - / 652 / 609 to 632;
  // the last with 512 x 2 in pairs 630, 256 x 4 in pairs 678)
  const bool few = rows * C <= sm_count;
  if (pieces / C < (few ? 1024 : 3000)) return launch_plan<TIn, TOut, 128, 8>(p, C, rows, sm_count, s);
  if (pieces / C < (few ? 4096 : 10000)) return launch_plan<TIn, TOut, 256, 4>(p, C, rows, sm_count, s);
  // The longest rows: not many more than 45 MB at a time, or their second read misses L2.  The plans above do not look
  // at that: 592 rows at a time are 60 MB at 50 257 bf16 entries and 95 MB just below 80 000, and the reads from
  // memory grow from 1.10 times the logits there over 1.31 (65 536) to 1.53 (2 300 rows: 104, 132, 171 us over 70, 92, 112 at
  // the copy rate; fp32 rows of half as many entries 97, 126, 163).
  while (C < kMaxCtas && sm_count / C * p.V * (int64_t)sizeof(TIn) > (int64_t(50) << 20)) C *= 2;
  return launch_plan<TIn, TOut, 960, 1>(p, C, rows, sm_count, s);
}

}  // namespace

cudaError_t launch_topk_kl(const void* logits, int dtype, int64_t B, int64_t T, int64_t V, int64_t ld,
                           const int32_t* tokens, const int32_t* window, const int32_t* rollout_len,
                           const int32_t* top_ids, const float* top_logprobs, const float* rest, int K,
                           float alpha, int kl_mode, int flags, void* grad, int grad_dtype, int64_t ld_grad,
                           float* kl, float* logratio, float* gsq, float* lse, int32_t* status,
                           int sm_count, cudaStream_t s) {
  TopkParams p = {};
  p.logits = logits;
  p.V = V;
  p.ld = ld;
  p.range = RowRange{(flags & ADWIN_RANGE_FULL) ? nullptr : window, rollout_len, B, T};
  p.window = window;
  p.rollout = rollout_len;
  p.tokens = tokens;
  p.top_ids = top_ids;
  p.top_logprobs = top_logprobs;
  p.rest = rest;
  p.K = K;
  p.alpha = alpha;
  p.forward = kl_mode == ADWIN_KL_FORWARD;
  p.zero_tail = (flags & ADWIN_ZERO_TAIL) != 0;
  p.grad = grad;
  p.ld_grad = ld_grad;
  p.kl = kl;
  p.logratio = logratio;
  p.gsq = gsq;
  p.lse = lse;
  p.status = status;
  p.limit_ns = handshake_wait_limit_ns();
  const int64_t rows = B * T;
  const bool out_bf = grad && grad_dtype == ADWIN_BF16;
  if (dtype == ADWIN_BF16)
    return out_bf || !grad ? launch<__nv_bfloat16, __nv_bfloat16>(p, rows, sm_count, s)
                           : launch<__nv_bfloat16, float>(p, rows, sm_count, s);
  return out_bf ? launch<float, __nv_bfloat16>(p, rows, sm_count, s) : launch<float, float>(p, rows, sm_count, s);
}

}  // namespace adwin
