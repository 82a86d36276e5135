// Divergence of the student from a teacher known by its K most likely alternatives and the mass
// outside them, with the gradient: one read of the student's logits, one write of the gradient.
//
// Categories c: the alternatives j = 1..K, each an entry id_j of the vocabulary, and the rest r,
//   P_j = exp(z_id_j - lse),   P_r = sum over all other entries of p_k,   Q_j, Q_r the teacher's:
//   reverse  KL = sum_c P_c (log P_c - log Q_c),    g_k = alpha p_k (D_c(k) - KL),   D_c = log P_c - log Q_c
//   forward  KL = sum_c Q_c (log Q_c - log P_c),    g_k = alpha (p_k - Q_c(k) p_k / P_c(k)).
// So every entry of the rest gets p_k times one coefficient of the row.  P_r is summed over the entries
// of the rest alone (1 - sum_j P_j would have no correct digit where the list holds nearly everything):
// a thread masks the listed entries out of the pieces they lie in, of which it has a list in shared
// memory, empty for most threads.  |g|^2 needs sum p_k^2 over the rest beside it.
//
// A row is read once: a thread fetches 16-byte pieces with cp.async into slots of its own in shared
// memory and takes them from there in both sweeps, so the copies need no barrier.  A slot that
// the second sweep has read is refilled at once with a piece of a row to come; what a CTA (or a cluster of
// them, a slice of the row each) has in flight is the ring's room beyond one row.  Between the sweeps
// the warps meet once, at the cluster's barrier, and each derives the row's scalars for itself.  One
// more warp looks the rows up, prepares the lists of the row after next, sums the few entries beside
// the 16-byte pieces and writes the row's outputs.
// Rows that no ring holds (kStream) are read twice.
#include "adwin_common.cuh"
#include "adwin_internal.h"
#include "exp_sums.cuh"
#include "row_list.cuh"

namespace adwin {
namespace {

constexpr int kGroup = 4;        // pieces a thread takes at a time
constexpr int kMaxCtas = 8;      // of a cluster

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
  int n, ring;               // slots of a row, slots of the ring
};

// What the threads have to know of a row.
struct RowInfo {
  const char* row;       // its logits, or null: no more rows
  char* out;             // its gradient, or null
  int64_t r;
  int64_t entry0;        // vocabulary index of the slice's first piece
  int head, tail;
  int np;                // pieces of the slice
  int y;
};

// The listed entries of a row.  Every entry is in the chain of one thread, that whose pieces hold it
// where there is one; an index that comes twice is found in its chain.
template <int TH>
struct TopList {
  int32_t id[ADWIN_TOP_MAX];      // -1: none
  float z[ADWIN_TOP_MAX], lq[ADWIN_TOP_MAX];
  int32_t slot[ADWIN_TOP_MAX];    // where it lies among its thread's pieces, or -1: not in this CTA's
  int16_t owner[ADWIN_TOP_MAX];   // the chain it is in, or -1
  int16_t next[ADWIN_TOP_MAX];
  int32_t first[TH];              // -1: an empty chain
  float lq_rest;
};

struct alignas(16) SumRecord {   // (written to a cluster's other CTAs in one piece)
  float m, s, q;   // reference, sum e, sum e^2 over entries of the rest
  float pad;
};

template <int TH>
struct TopkShared {
  static constexpr int kWarps = TH / 32 + 1;
  RowList list;
  RowInfo info[4];
  TopList<TH> lists[3];
  SumRecord rec[2][kMaxCtas * kWarps];
};
static_assert(alignof(TopkShared<128>) == 16 && sizeof(SumRecord) == 16, "records are stored 16 bytes at a time");

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most `pending` groups of this thread's copies are in flight (the instruction
// takes a constant).
__device__ __forceinline__ void copies_wait(int pending) {
#define ADWIN_WAIT(n) case n: asm volatile("cp.async.wait_group " #n ";" ::: "memory"); break;
  switch (pending) {
    ADWIN_WAIT(1) ADWIN_WAIT(2) ADWIN_WAIT(3) ADWIN_WAIT(4) ADWIN_WAIT(5) ADWIN_WAIT(6) ADWIN_WAIT(7)
    ADWIN_WAIT(8) ADWIN_WAIT(9) ADWIN_WAIT(10) ADWIN_WAIT(11) ADWIN_WAIT(12) ADWIN_WAIT(13)
    ADWIN_WAIT(14) ADWIN_WAIT(15) ADWIN_WAIT(16) ADWIN_WAIT(17) ADWIN_WAIT(18) ADWIN_WAIT(19)
    ADWIN_WAIT(20) ADWIN_WAIT(21) ADWIN_WAIT(22) ADWIN_WAIT(23) ADWIN_WAIT(24) ADWIN_WAIT(25)
    default: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
  }
#undef ADWIN_WAIT
}
__device__ __forceinline__ uint4 read16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr)
               : "memory");
  return v;
}

template <typename TIn>
__device__ __forceinline__ uint4 masked_piece() {
  constexpr uint32_t w = sizeof(TIn) == 2 ? 0xff80ff80u : 0xff800000u;   // -infinity
  return make_uint4(w, w, w, w);
}
template <typename TIn>
__device__ __forceinline__ void mask_entry(uint4& v, int e) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(TIn) == 4) {
      if (e == i) w[i] = 0xff800000u;
    } else {
      if (e == 2 * i) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
      if (e == 2 * i + 1) w[i] = (w[i] & 0xffffu) | 0xff800000u;
    }
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
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
  __device__ __forceinline__ void add(f2_t z) {
    const f2_t e = ex2_2(mul2(add2(z, splat2(-m)), splat2(kLog2e)));
    S = add2(S, e);
    Q = fma2(e, e, Q);
  }
};

// Scalars of a row, the same in every warp.
struct TopScalars {
  float M, ln_s, inv_s;   // reference, log and inverse of the whole sum against it
  float kl, d_rest;
  // g_k = alpha c_rest exp(z_k - m_rest) for entries of the rest: against their own largest, for
  // the forward divergence divides by their mass, however far that is below the listed entries'
  float m_rest, c_rest;
  float gsq_rest;         // sum (g_k / alpha)^2 over them
};
// Gradient at a listed entry, before alpha.
__device__ __forceinline__ float listed_grad(const TopScalars& t, float z, float lq, bool forward) {
  const float p = exp_below(z, t.M) * t.inv_s;
  if (forward) return p - expf(lq);
  return p == 0.f ? 0.f : p * ((((z - t.M) - t.ln_s) - lq) - t.kl);
}

template <typename TIn, typename TOut, int TH, bool STREAM>
struct TopkCta {
  static constexpr int N = Elem<TIn>::N, NP = Pairs<TIn>::NP;
  static constexpr int kWarps = TH / 32 + 1;
  const TopkParams& p;
  TopkShared<TH>& sh;
  const uint32_t ring;         // shared address of the slots
  const int C, me, tid, lane, warp;
  int64_t rows, cursor, step;

  // Next row of this cluster becomes info[o % 4]; one warp.
  __device__ __forceinline__ void look_up(int o) {
    int64_t r = -1;
    while (cursor < rows) {
      r = sh.list.row(p.range, cursor);
      cursor += step;
      if (r >= 0) break;
    }
    RowInfo i = {};
    i.r = r;
    if (r >= 0) {
      i.row = static_cast<const char*>(p.logits) + (size_t)r * p.ld * sizeof(TIn);
      const RowPieces rp = RowPieces::of<TIn>(i.row, p.V);
      const int64_t per = (rp.pieces + C - 1) / C, first = per * me < rp.pieces ? per * me : rp.pieces;
      i.np = (int)(first + per < rp.pieces ? per : rp.pieces - first);
      i.entry0 = rp.head + first * N;
      i.head = me == 0 ? rp.head : 0;
      i.tail = me == C - 1 ? rp.tail : 0;
      i.y = p.tokens[r];
      if (p.grad) {
        const int64_t b = r / p.range.T;
        const RowRange w = {p.window, p.rollout, p.range.B, p.range.T};
        if (r - b * p.range.T < w.end(b)) i.out = static_cast<char*>(p.grad) + (size_t)r * p.ld_grad * sizeof(TOut);
      }
    }
    if (lane == 0) sh.info[o & 3] = i;
    __syncwarp();
  }

  // The list of the row of info[o % 4] into lists[o % 3]; one warp.
  __device__ __forceinline__ void prepare(int o) {
    TopList<TH>& l = sh.lists[o % 3];
    const RowInfo& i = sh.info[o & 3];
    const int K = p.K;
    for (int j = lane; j < K; j += 32)      // (the list that was here)
      if (l.owner[j] >= 0) l.first[l.owner[j]] = -1;
    __syncwarp();
    double left = 0.0;
    for (int j = lane; j < K; j += 32) {
      int32_t id = i.row ? p.top_ids[i.r * K + j] : -1;
      if (id < -1 || (int64_t)id >= p.V) {
        if (me == 0) atomicOr(p.status, (int32_t)ADWIN_DEV_TOKEN_RANGE);
        id = -1;
      }
      int owner = -1, slot = -1;
      if (id >= 0) {
        const int64_t e = (int64_t)id - i.entry0;
        if (e >= 0 && e < (int64_t)i.np * N) {
          owner = (int)(e / N % TH);
          slot = (int)(e / N / TH);
        } else {
          owner = id % TH;   // (any thread)
        }
      }
      l.id[j] = id;
      l.lq[j] = id >= 0 ? p.top_logprobs[i.r * K + j] : 0.f;
      l.z[j] = id >= 0 ? Elem<TIn>::load1(i.row, id) : 0.f;
      l.slot[j] = slot;
      l.owner[j] = (int16_t)owner;
      if (owner >= 0) l.next[j] = (int16_t)atomicExch(&l.first[owner], j);   // (the order of a chain does not matter)
    }
    __syncwarp();
    uint32_t again = 0;
    for (int j = lane, bit = 0; j < K; j += 32, ++bit) {
      if (l.owner[j] < 0) continue;
      for (int k = l.first[l.owner[j]]; k >= 0; k = l.next[k])
        if (k < j && l.id[k] == l.id[j]) again |= 1u << bit;
    }
    __syncwarp();
    for (int j = lane, bit = 0; j < K; j += 32, ++bit) {
      if (again >> bit & 1) {
        l.id[j] = -1;
        l.slot[j] = -1;
        if (me == 0) atomicOr(p.status, (int32_t)ADWIN_DEV_TOKEN_RANGE);
      }
      if (l.id[j] >= 0 && !p.rest) left += exp((double)l.lq[j]);
    }
    float lqr = 0.f;
    if (p.rest) {
      lqr = i.row ? p.rest[i.r] : 0.f;
    } else {
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) left += __shfl_xor_sync(0xffffffffu, left, s);
      lqr = (float)log(fmax(1.0 - left, 5.9604644775390625e-8));   // 2^-24
    }
    if (lane == 0) l.lq_rest = lqr;
    __syncwarp();
  }

  // An entry beside the slice's pieces that this lane of the extra warp holds, or -1.
  __device__ __forceinline__ int64_t edge_of(const RowInfo& i) const {
    if (lane < i.head) return lane;
    if (lane >= 16 && lane - 16 < i.tail) return p.V - i.tail + (lane - 16);
    return -1;
  }
  __device__ __forceinline__ int listed(const TopList<TH>& l, int64_t id) const {
    int found = -1;
    for (int j = 0; j < p.K; ++j)
      if (l.id[j] == (int32_t)id) found = j;
    return found;
  }

  // Hands a warp's sum to every CTA of the cluster.
  __device__ __forceinline__ void publish(int par, float m, float s, float q) {
    SumRecord* mine = &sh.rec[par][me * kWarps + warp];
    if (C == 1) {
      if (lane == 0) *mine = SumRecord{m, s, q, 0.f};
    } else if (lane < C) {
      remote_store4(map_to_rank(smem_u32(mine), (uint32_t)lane), m, s, q, 0.f);
    }
  }
  __device__ __forceinline__ void meet() const {
    if (C == 1) __syncthreads(); else cluster_sync_all();
  }

  // Every warp for itself, the same arithmetic in the same order.
  __device__ __forceinline__ TopScalars scalars(int par, const TopList<TH>& l, float& gsq_listed) const {
    float m = kLowest;
    const int n = C * kWarps;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, sh.rec[par][i].m);
    m = warp_max(m);
    float s = 0.f, q = 0.f;
    for (int i = lane; i < n; i += 32) {
      const SumRecord r = sh.rec[par][i];
      const float w = exp_below(r.m, m);
      s = fmaf(w, r.s, s);
      q = fmaf(w * w, r.q, q);
    }
    s = lane_sum(s);
    q = lane_sum(q);
    float z[ADWIN_TOP_MAX / 32], lq[ADWIN_TOP_MAX / 32];
    float M = m;
#pragma unroll
    for (int k = 0; k < ADWIN_TOP_MAX / 32; ++k) {
      const int j = lane + 32 * k;
      const bool there = j < p.K && l.id[j] >= 0;
      z[k] = there ? l.z[j] : -INFINITY;
      lq[k] = there ? l.lq[j] : -INFINITY;
      M = fmaxf(M, z[k]);
    }
    M = warp_max(M);
    float st = 0.f;
#pragma unroll
    for (int k = 0; k < ADWIN_TOP_MAX / 32; ++k) st += exp_below(z[k], M);   // (-inf: 0, NaN stays)
    st = lane_sum(st);
    TopScalars t;
    t.M = M;
    const float wr = exp_below(m, M), sum = fmaf(wr, s, st);
    t.ln_s = logf(sum);
    t.inv_s = 1.f / sum;
    const float pr = wr * s * t.inv_s, lqr = l.lq_rest;
    const float lpr = s > 0.f ? (m - M) + (logf(s) - t.ln_s) : -INFINITY;
    t.d_rest = lpr - lqr;
    t.m_rest = m;
    float kl = 0.f;
#pragma unroll
    for (int k = 0; k < ADWIN_TOP_MAX / 32; ++k) {
      const int j = lane + 32 * k;
      if (j >= p.K || l.id[j] < 0) continue;
      const float lp = (z[k] - M) - t.ln_s, pj = exp_below(z[k], M) * t.inv_s, qj = expf(lq[k]);
      if (p.forward) kl += qj == 0.f ? 0.f : qj * (lq[k] - lp);
      else kl += pj == 0.f ? 0.f : pj * (lp - lq[k]);
    }
    kl = lane_sum(kl);
    t.c_rest = 0.f;   // (no entry is left, or none with any mass)
    if (p.forward) {
      const float qr = expf(lqr);
      kl += qr == 0.f ? 0.f : qr * -t.d_rest;
      if (s != 0.f) t.c_rest = wr * t.inv_s - qr / s;
    } else if (s != 0.f) {
      kl += pr == 0.f ? 0.f : pr * t.d_rest;
      t.c_rest = wr == 0.f ? 0.f : (t.d_rest - kl) * (wr * t.inv_s);
    }
    t.gsq_rest = t.c_rest * t.c_rest * q;
    t.kl = kl;
    gsq_listed = 0.f;
    if (warp == kWarps - 1) {
#pragma unroll
      for (int k = 0; k < ADWIN_TOP_MAX / 32; ++k) {
        const int j = lane + 32 * k;
        if (j >= p.K || l.id[j] < 0) continue;
        const float g = listed_grad(t, z[k], lq[k], p.forward);
        gsq_listed = fmaf(g, g, gsq_listed);
      }
      gsq_listed = lane_sum(gsq_listed);
    }
    return t;
  }

  // The warp beside the sweeps.
  __device__ __forceinline__ void extra_warp() {
    for (int i = 0;; ++i) {
      const RowInfo& info = sh.info[i & 3];
      if (!info.row) break;
      const TopList<TH>& l = sh.lists[i % 3];
      const int64_t e = edge_of(info);
      const float z = e >= 0 ? Elem<TIn>::load1(info.row, e) : -INFINITY;
      const int j = e >= 0 ? listed(l, e) : -1;
      {
        const float zr = j >= 0 ? -INFINITY : z, m = fmaxf(warp_max(zr), kLowest), x = exp_below(zr, m);
        publish(i & 1, m, lane_sum(x), lane_sum(x * x));
      }
      meet();
      float gl;
      const TopScalars t = scalars(i & 1, l, gl);
      if (info.out && e >= 0) {
        const float g = j >= 0 ? listed_grad(t, z, l.lq[j], p.forward) : t.c_rest * exp_below(z, t.m_rest);
        Elem<TOut>::store1(info.out, e, p.alpha * g);
      }
      if (me == 0) {
        const int y = info.y;
        const bool y_valid = y >= 0 && (int64_t)y < p.V;
        int jy = -1;
        for (int k = lane; k < p.K; k += 32)
          if (y_valid && l.id[k] == y) jy = k;
        jy = __reduce_max_sync(0xffffffffu, jy);
        if (lane == 0) {
          const float lse = t.M + t.ln_s;
          p.kl[info.r] = t.kl;
          p.logratio[info.r] = !y_valid ? __int_as_float(0x7fc00000)
                               : jy >= 0 ? ((l.z[jy] - t.M) - t.ln_s) - l.lq[jy] : t.d_rest;
          if (p.gsq) p.gsq[info.r] = p.alpha * p.alpha * (t.gsq_rest + gl);
          if (p.lse) p.lse[info.r] = lse;
          int bits = 0;
          if (!y_valid) bits |= ADWIN_DEV_TOKEN_RANGE;
          if (!isfinite(lse) || !isfinite(t.kl)) bits |= ADWIN_DEV_NONFINITE;
          if (bits) atomicOr(p.status, bits);
        }
      }
      look_up(i + 3);
      prepare(i + 2);
    }
  }

  // Asks for slot j of the row of `info`; position q of the ring.
  __device__ __forceinline__ void fetch(const RowInfo& info, int j, int pos) const {
    const int piece = j * TH + tid;
    if (info.row && piece < info.np &&
        ADWIN_CHK(pos >= 0 && pos < p.ring && info.entry0 + (int64_t)(piece + 1) * N <= p.V, p.status))
      copy16(ring + (uint32_t)(pos * TH + tid) * 16u, info.row + (size_t)info.entry0 * sizeof(TIn) + (size_t)piece * 16);
    copies_commit();
  }

  __device__ __forceinline__ void sweeps() {
    const int n = p.n, R = p.ring;
    int base = 0;   // ring position of the row's slot 0
    if (!STREAM) {
      for (int q = 0; q < R; ++q) fetch(sh.info[q / n], q % n, q);   // (R <= 2 n)
    }
    for (int i = 0;; ++i) {
      const RowInfo& info = sh.info[i & 3];
      if (!info.row) break;
      const TopList<TH>& l = sh.lists[i % 3];
      const int np = info.np;
      const uint4* src = reinterpret_cast<const uint4*>(info.row + (size_t)info.entry0 * sizeof(TIn));
      const int slots = STREAM ? (np + TH - 1) / TH : n;
      // which of this thread's slots hold listed entries (with more than 32 slots, which may)
      const int chain = l.first[tid];
      uint32_t marked = 0;
      for (int j = chain; j >= 0; j = l.next[j])
        if (l.slot[j] >= 0) marked |= 1u << (l.slot[j] & 31);

      auto take = [&](int j) {
        const int piece = j * TH + tid;
        if (j >= slots || piece >= np) return masked_piece<TIn>();
        if (STREAM) return ADWIN_CHK(info.entry0 + (int64_t)(piece + 1) * N <= p.V, p.status)
                               ? __ldcg(src + piece) : masked_piece<TIn>();
        int pos = base + j;
        if (pos >= R) pos -= R;
        return read16(ring + (uint32_t)(pos * TH + tid) * 16u);
      };

      RestSum acc;
      acc.reset();
      for (int j0 = 0; j0 < slots; j0 += kGroup) {
        // copies committed so far: those of i n + R slots
        if (!STREAM) copies_wait(R - (j0 + kGroup < n ? j0 + kGroup : n));
        uint4 v[kGroup];
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          v[k] = take(j0 + k);
          if (marked >> ((j0 + k) & 31) & 1) {
            for (int j = chain; j >= 0; j = l.next[j])
              if (l.slot[j] == j0 + k) mask_entry<TIn>(v[k], (int)((l.id[j] - info.entry0) % N));
          }
        }
        acc.raise(group_max(v, static_cast<TIn*>(nullptr)));
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          f2_t z[NP];
          Pairs<TIn>::make(v[k], z);
#pragma unroll
          for (int x = 0; x < NP; ++x) acc.add(z[x]);
        }
      }
      {
        const float m = warp_max(acc.m), w = exp_below(acc.m, m);
        publish(i & 1, m, lane_sum(w * hsum2(acc.S)), lane_sum(w * w * hsum2(acc.Q)));
      }
      meet();
      float unused;
      const TopScalars t = scalars(i & 1, l, unused);

      char* out = info.out ? info.out + (size_t)info.entry0 * sizeof(TOut) : nullptr;
      constexpr int kOutAlign = N * sizeof(TOut) < 16 ? (int)(N * sizeof(TOut)) : 16;
      const bool wide = (reinterpret_cast<uintptr_t>(out) & (kOutAlign - 1)) == 0;
      const f2_t neg_m = splat2(-t.m_rest), coef = splat2(p.alpha * t.c_rest);
      for (int j = 0; j < slots; ++j) {
        const int piece = j * TH + tid;
        if (out && piece < np) {
          const uint4 v = take(j);
          f2_t z[NP], g[NP];
          Pairs<TIn>::make(v, z);
#pragma unroll
          for (int x = 0; x < NP; ++x) g[x] = mul2(coef, ex2_2(mul2(add2(z[x], neg_m), splat2(kLog2e))));
          if (marked >> (j & 31) & 1) {
            for (int k = chain; k >= 0; k = l.next[k]) {
              if (l.slot[k] != j) continue;
              const int at = (int)((l.id[k] - info.entry0) % N);
              const float gl = p.alpha * listed_grad(t, l.z[k], l.lq[k], p.forward);
#pragma unroll
              for (int x = 0; x < NP; ++x) {
                float a, b;
                upk2(g[x], a, b);
                g[x] = pk2(at == 2 * x ? gl : a, at == 2 * x + 1 ? gl : b);
              }
            }
          }
          if (wide) {
            store_pairs<TOut>(out + (size_t)piece * N * sizeof(TOut), g);
          } else {
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              float a, b;
              upk2(g[x], a, b);
              Elem<TOut>::store1(out, (int64_t)piece * N + 2 * x, a);
              Elem<TOut>::store1(out, (int64_t)piece * N + 2 * x + 1, b);
            }
          }
        }
        if (!STREAM) {
          int o = i, jj = j + R;
          while (jj >= n) {
            jj -= n;
            ++o;
          }
          int pos = base + j;
          if (pos >= R) pos -= R;
          fetch(sh.info[o & 3], jj, pos);
        }
      }
      base += n;
      while (base >= R) base -= R;
    }
    if (!STREAM) copies_wait(0);
  }
};

template <typename TIn, typename TOut, int TH, int CTAS, bool STREAM>
__global__ void __launch_bounds__(TH + 32, CTAS) topk_kl_kernel(const TopkParams p) {
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
  for_rows_outside(p.range, [&](int64_t r) {
    p.kl[r] = 0.f;
    p.logratio[r] = 0.f;
    if (p.gsq) p.gsq[r] = 0.f;
    if (p.lse) p.lse[r] = 0.f;
  });
  for (int j = tid; j < 3 * TH; j += blockDim.x) sh.lists[j / TH].first[j % TH] = -1;
  for (int j = tid; j < 3 * ADWIN_TOP_MAX; j += blockDim.x) sh.lists[j / ADWIN_TOP_MAX].owner[j % ADWIN_TOP_MAX] = -1;
  __syncthreads();
  TopkCta<TIn, TOut, TH, STREAM> cta = {p, sh, smem_u32(smem) + (uint32_t)((sizeof(TopkShared<TH>) + 15) & ~size_t(15)),
                                        C, me, tid, tid & 31, warp, sh.list.count(p.range),
                                        (int64_t)(blockIdx.x / C), (int64_t)(gridDim.x / C)};
  if (warp == TH / 32) {
    for (int o = 0; o < 3; ++o) cta.look_up(o);
    cta.prepare(0);
    cta.prepare(1);
  }
  cta.meet();   // (the CTAs of a cluster are all there before anything is written to one)
  if (warp == TH / 32) cta.extra_warp(); else cta.sweeps();
  if (p.zero_tail && p.grad) {
    const RowRange w = {p.window, p.rollout, p.range.B, p.range.T};
    zero_rows_outside<TOut>(w, p.grad, p.ld_grad, p.V);
  }
}

template <typename TIn, typename TOut, int TH, int CTAS, bool STREAM>
cudaError_t launch_plan(const TopkParams& p, int C, int64_t rows, int sm_count, cudaStream_t s) {
  const size_t base = (sizeof(TopkShared<TH>) + 15) & ~size_t(15);
  // a CTA's whole share, the same for every launch of this kernel
  constexpr size_t share = (size_t)(228 * 1024 / CTAS - 1024) & ~size_t(15);
  const size_t smem = STREAM ? base : base + (size_t)p.ring * TH * 16;
  if (smem > share) return cudaErrorInvalidValue;
  auto kernel = topk_kl_kernel<TIn, TOut, TH, CTAS, STREAM>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)share);
  if (e != cudaSuccess) return e;
  int64_t clusters = (int64_t)sm_count * CTAS / C;
  if (clusters > rows) clusters = rows;
  return launch_chained(kernel, (unsigned)(clusters * C), TH + 32, smem, C, s, p);
}

template <typename TIn, typename TOut>
cudaError_t launch(TopkParams p, int64_t rows, int sm_count, cudaStream_t s) {
  const int64_t pieces = (p.V + Elem<TIn>::N - 1) / Elem<TIn>::N;
  auto room = [](size_t th, size_t ctas) {
    const size_t base = (th == 128 ? sizeof(TopkShared<128>) : th == 256 ? sizeof(TopkShared<256>) : sizeof(TopkShared<512>));
    return (int)((228 * 1024 / ctas - 1024 - 32 - base) / (th * 16));
  };
  // few rows: several CTAs to a row, as long as each has two slots to a thread
  int C = 1;
  while (C < kMaxCtas && rows * C * 2 <= sm_count && pieces >= (int64_t)C * 2 * 1024) C *= 2;
  auto fit = [&](int th, int ctas) {
    p.n = (int)((pieces + C - 1) / C + th - 1) / th;
    if (p.n < 1) p.n = 1;
    p.ring = room(th, ctas) < 2 * p.n ? room(th, ctas) : 2 * p.n;
    if (p.ring > 25) p.ring = 25;
    // the ring must hold a row and keep some of the next in flight
    return p.ring >= p.n + (p.n + 3) / 4;
  };
  if (fit(128, 6)) return launch_plan<TIn, TOut, 128, 6, false>(p, C, rows, sm_count, s);
  if (fit(256, 3)) return launch_plan<TIn, TOut, 256, 3, false>(p, C, rows, sm_count, s);
  for (; C <= kMaxCtas; C *= 2)
    if (fit(512, 1)) return launch_plan<TIn, TOut, 512, 1, false>(p, C, rows, sm_count, s);
  return launch_plan<TIn, TOut, 512, 1, true>(p, 1, rows, sm_count, s);
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
  const int64_t rows = B * T;
  const bool out_bf = grad && grad_dtype == ADWIN_BF16;
  if (dtype == ADWIN_BF16)
    return out_bf || !grad ? launch<__nv_bfloat16, __nv_bfloat16>(p, rows, sm_count, s)
                           : launch<__nv_bfloat16, float>(p, rows, sm_count, s);
  return out_bf ? launch<float, __nv_bfloat16>(p, rows, sm_count, s) : launch<float, float>(p, rows, sm_count, s);
}

}  // namespace adwin
