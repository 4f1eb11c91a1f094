// Verification of drafted tokens against the policy's rows (speculative decoding) with given random
// numbers: which drafts are accepted, the token drawn behind them, and the log-probs of both.
//
// Accepting compares u q(x) with p(x), and the draw finds where a running sum passes u times its
// total: both turn on the last bits of sums over the vocabulary, and another summation order would
// now and then emit another token. So probabilities, sums and running sums are held in 64 bits, with
// exponentials good to 2e-14; fused multiply-adds in 64 bits run at the 32-bit rate here, and an
// exponential costs about twice what the 32-bit path with the transcendental unit does.
//
// Three kernels: the maximum and sum of exponentials of every row that a sequence may need, in parts
// where rows are few; the weights' sums over cells of 64 chunks of the row each sequence draws from
// (each workgroup first decides, from the rows' sums, where its sequence stops); and the draw: the
// cell where the running sum passes, then the entry.
#include "verify.h"

#include <algorithm>

#include "dppo_device.h"
#include "f64_math.h"
#include "row_split.h"

namespace dppo {

namespace {

constexpr int kStatsNT = 256;
constexpr int kCellNT = 256;
constexpr int kPickNT = 256;
constexpr int kMaxParts = 16;
constexpr int64_t kStatsRows = 512;   // rows of a launch of the statistics

template <typename Tin>
__device__ __forceinline__ float entry_value(const Tin* p, int64_t i) {
  if constexpr (sizeof(Tin) == 2) return bf16_to_f32(p[i]);
  else return p[i];
}

template <typename Tin, class W>
__device__ __forceinline__ void unpack(const W& r, float (&x)[16 / sizeof(Tin)]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(Tin) == 2) {
      x[2 * k] = bf16_lo(r[k]);
      x[2 * k + 1] = bf16_hi(r[k]);
    } else {
      x[k] = __uint_as_float(r[k]);
    }
  }
}

__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int b) {
  if (!a.num) return a.D;
  const int n = a.num[b];
  return n < 0 ? 0 : (n > a.D ? a.D : n);
}
template <typename Tin>
__device__ __forceinline__ const Tin* target_row(const VerifyArgs& a, int64_t b, int64_t i) {
  return (const Tin*)a.target + b * a.target_seq + i * a.target_row;
}
template <typename Tin>
__device__ __forceinline__ const Tin* draft_row(const VerifyArgs& a, int64_t b, int64_t i) {
  return (const Tin*)a.draft + b * a.draft_seq + i * a.draft_row;
}

// Joins (maximum, sum of 2^((z - maximum) t2e)) pairs; maxima in the logits' units. A sum that is NaN
// stays so.
__device__ __forceinline__ void join(double& m, double& s, double m2, double s2, double t2e) {
  const double M = fmax(m, m2);
  const double fa = m == M ? 1.0 : exp2_f64((m - M) * t2e);
  const double fb = m2 == M ? 1.0 : exp2_f64((m2 - M) * t2e);
  s = s * fa + s2 * fb;
  m = M;
}

// A row's normaliser from its parts; NaN for a row that cannot be evaluated.
__device__ __forceinline__ VerifyNorm row_norm(const VerifyArgs& a, int64_t b, int64_t i, int kind) {
  const double* st = a.stats + ((i * a.B + b) * 2 + kind) * a.parts * 2;
  double m = st[0], s = st[1];
  for (int p = 1; p < a.parts; ++p) join(m, s, st[2 * p], st[2 * p + 1], a.t2e);
  return {m, s > 0.0 && s < INFINITY && m < INFINITY ? log2_f64(s) : (double)__builtin_nanf("")};
}
// log2 of an entry's probability.
__device__ __forceinline__ double log2_prob(const VerifyArgs& a, const VerifyNorm& n, float z) {
  return __builtin_fma((double)z - n.m, a.t2e, -n.log2s);
}

// Where sequence b stops among its first n drafts, by one wave; every lane returns the same. With
// `write`, the accepted drafts and their log-probs go to the outputs. (Lanes behind the stop may read
// statistics that were never computed; the first lane that stops decides.)
template <typename Tin>
__device__ __forceinline__ VerifyDraw decide(const VerifyArgs& a, int b, int n, bool write) {
  const int lane = threadIdx.x & 63;
  VerifyDraw d{};
  d.pos = n;
  d.mode = kDrawTarget;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    bool accept = true, bad = false;
    VerifyNorm np{}, nq{};
    float out = 0.0f;
    int64_t x = -1;
    if (i < n) {
      x = a.ids[(int64_t)b * a.D + i];
      np = row_norm(a, b, i, 0);
      if (a.draft) nq = row_norm(a, b, i, 1);
      bad = x < 0 || x >= a.V || np.log2s != np.log2s || nq.log2s != nq.log2s;
      accept = false;
      if (!bad) {
        const double lp = log2_prob(a, np, entry_value(target_row<Tin>(a, b, i), x));
        const double q = a.draft ? exp2_f64(log2_prob(a, nq, entry_value(draft_row<Tin>(a, b, i), x))) : 1.0;
        accept = (double)a.u[(int64_t)b * a.D + i] * q < exp2_f64(lp);
        out = (float)(lp * kLn2F64);
      }
    }
    const uint64_t stops = __ballot(!accept);
    const int stop = stops ? __builtin_ctzll(stops) : 64;
    if (write && i < n && lane < stop) {
      a.tokens[(int64_t)b * (a.D + 1) + i] = x;
      a.logp[(int64_t)b * (a.D + 1) + i] = out;
    }
    if (stop < 64) {
      d.pos = i0 + stop;
      d.p = {__shfl(np.m, stop, 64), __shfl(np.log2s, stop, 64)};
      d.q = {__shfl(nq.m, stop, 64), __shfl(nq.log2s, stop, 64)};
      d.mode = __shfl((int)bad, stop, 64) ? kDrawBad : (a.draft ? kDrawResidual : kDrawWithout);
      return d;
    }
  }
  return d;
}

// One part of one row's statistics per workgroup, for the positions [i0, i1); positions outermost.
// Sequences that stop before i0 (their statistics are complete: an earlier launch) are skipped.
template <typename Tin>
__global__ __launch_bounds__(kStatsNT) void verify_stats(VerifyArgs a, int i0, int i1) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int NT = kStatsNT;
  constexpr int U = 4;
  constexpr int NW = NT / 64;
  constexpr int kOff = 0x7fffff00;
  __shared__ double red[2 * NW];
  __shared__ int alive;
  const int tid = threadIdx.x;
  const int kinds = a.draft ? 2 : 1;
  const int64_t items = (int64_t)(i1 - i0) * a.B * kinds * a.parts;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int part = (int)(item % a.parts);
    const int64_t rest = item / a.parts;
    const int kind = (int)(rest % kinds);
    const int b = (int)((rest / kinds) % a.B);
    const int i = i0 + (int)((rest / kinds) / a.B);
    const int drafts = drafts_of(a, b);
    if (i + kind > drafts) continue;                 // uniform: not a row of this sequence
    const int64_t at = (int64_t)i * a.B + b;
    const Tin* z = kind ? draft_row<Tin>(a, b, i) : target_row<Tin>(a, b, i);
    const RowSplit sp = split_row(z, a.V);
    const int c0 = (int)((int64_t)sp.nfull * part / a.parts);
    const int n = (int)((int64_t)sp.nfull * (part + 1) / a.parts) - c0;
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead + (int64_t)c0 * E, n * 16);
    u32x4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = buf_load16<kAuxLast>(rz, u * NT + tid < n ? (u * NT + tid) * 16 : kOff, 0);
    if (i0 > 0) {
      __syncthreads();                               // the last item's flag is read
      if (tid < 64) {
        const bool on = decide<Tin>(a, b, i0, false).mode == kDrawTarget;
        if (tid == 0) alive = on;
      }
      __syncthreads();
      if (!alive) continue;
    }
    float m = -INFINITY;                             // this thread's maximum
    double s = 0.0, ref = 0.0;                       // ref: m, or 0 while that is -inf
    auto add = [&](const auto& x, float cm) {
      if (cm > m) {
        s *= exp2_f64(((double)m - (double)cm) * a.t2e);
        m = cm;
        ref = cm;
      }
      // the difference first: a product with a far logit (a mask of the type's lowest value) has no
      // fraction left
#pragma unroll
      for (int j = 0; j < (int)(sizeof(x) / 4); ++j) s += exp2_f64(((double)x[j] - ref) * a.t2e);
    };
    if (part == 0 && tid < sp.nedge) {
      const float x[1] = {entry_value(z, sp.entry<E>(tid))};
      add(x, x[0]);
    }
    for (int base = 0; base < n; base += U * NT) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = base + u * NT + tid;
        float x[E];
        unpack<Tin>(r[u], x);
        r[u] = buf_load16<kAuxLast>(rz, c + U * NT < n ? (c + U * NT) * 16 : kOff, 0);
        if (c < n) {
          float cm = max3(x[0], x[1], x[2]);
          if constexpr (E == 8) cm = max3(cm, max3(x[3], x[4], x[5]), max3(x[6], x[7], x[7]));
          else cm = fmaxf(cm, x[3]);
          add(x, cm);
        }
      }
    }
    double md = m;
    {
      // the wave's maximum, then one exponential per thread (NaN sums stay NaN)
      const double M = wave_max_f64(md);
      s = wave_sum_f64(md == M ? s : s * exp2_f64((md - M) * a.t2e));
      md = M;
    }
    __syncthreads();                                 // the last item's partials are read
    if ((tid & 63) == 0) {
      red[tid >> 6] = md;
      red[NW + (tid >> 6)] = s;
    }
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < NW; ++w) join(md, s, red[w], red[NW + w], a.t2e);
      double* out = a.stats + ((at * 2 + kind) * a.parts + part) * 2;
      out[0] = md;
      out[1] = s;
    }
  }
}

// Weights of the E entries from entry e0 on (a whole chunk of the target's row).
template <typename Tin>
__device__ __forceinline__ void chunk_weights(const VerifyArgs& a, const VerifyDraw& d, int mode, const Tin* p,
                                              const Tin* q, int x, int e0, double (&w)[16 / sizeof(Tin)]) {
  constexpr int E = 16 / (int)sizeof(Tin);
  float z[E];
  unpack<Tin>(*(const u32x4*)(p + e0), z);
#pragma unroll
  for (int j = 0; j < E; ++j) w[j] = exp2_f64(log2_prob(a, d.p, z[j]));
  if (mode == kDrawResidual) {
    if (((uintptr_t)(q + e0) & 15) == 0) {
      unpack<Tin>(*(const u32x4*)(q + e0), z);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) z[j] = entry_value(q, e0 + j);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = fmax(w[j] - exp2_f64(log2_prob(a, d.q, z[j])), 0.0);
  } else if (mode == kDrawWithout) {
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = e0 + j == x ? 0.0 : w[j];
  }
}
template <typename Tin>
__device__ __forceinline__ double entry_weight(const VerifyArgs& a, const VerifyDraw& d, int mode, const Tin* p,
                                               const Tin* q, int x, int e) {
  double w = exp2_f64(log2_prob(a, d.p, entry_value(p, e)));
  if (mode == kDrawResidual) w = fmax(w - exp2_f64(log2_prob(a, d.q, entry_value(q, e))), 0.0);
  else if (mode == kDrawWithout && e == x)
    w = 0.0;
  return w;
}

// Cell 0 holds the entries before the row's whole chunks, cell c the 64 chunks from 64 (c - 1) on, the
// last cell the entries behind them. A lane's entries of a cell: `count` of them from `first` on.
struct CellSpan {
  int first, count;
};
template <typename Tin>
__device__ __forceinline__ CellSpan cell_span(const RowSplit& sp, int V, int cells, int cell, int lane) {
  constexpr int E = 16 / (int)sizeof(Tin);
  if (cell == 0) return {lane, lane < sp.lead ? 1 : 0};
  if (cell == cells - 1) {
    const int e = sp.lead + sp.nfull * E + lane;
    return {e, e < V ? 1 : 0};
  }
  const int c = (cell - 1) * 64 + lane;
  return {sp.lead + c * E, c < sp.nfull ? E : 0};
}
template <typename Tin>
__device__ __forceinline__ void span_weights(const VerifyArgs& a, const VerifyDraw& d, int mode, const Tin* p,
                                             const Tin* q, int x, const CellSpan& s, double (&w)[16 / sizeof(Tin)]) {
  constexpr int E = 16 / (int)sizeof(Tin);
  if (s.count == E) {
    chunk_weights(a, d, mode, p, q, x, s.first, w);
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = 0.0;
    if (s.count == 1) w[0] = entry_weight(a, d, mode, p, q, x, s.first);
  }
}

// The sum of a cell's weights, by one wave.
template <typename Tin>
__device__ __forceinline__ double cell_sum(const VerifyArgs& a, const VerifyDraw& d, int mode, const Tin* p,
                                           const Tin* q, int x, const RowSplit& sp, int cell) {
  constexpr int E = 16 / (int)sizeof(Tin);
  double w[E];
  span_weights(a, d, mode, p, q, x, cell_span<Tin>(sp, a.V, a.cells, cell, threadIdx.x & 63), w);
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < E; ++j) s += w[j];
  return wave_sum_f64(s);
}

template <typename Tin>
__global__ __launch_bounds__(kCellNT) void verify_cells(VerifyArgs a) {
  __shared__ VerifyDraw ds;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  for (int64_t item = blockIdx.x; item < (int64_t)a.B * a.draw_parts; item += gridDim.x) {
    const int b = (int)(item / a.draw_parts);
    const int part = (int)(item % a.draw_parts);
    __syncthreads();
    if (wave == 0) {
      const int n = drafts_of(a, b);
      VerifyDraw d = decide<Tin>(a, b, n, part == 0);
      if (d.mode == kDrawTarget) {
        d.p = row_norm(a, b, n, 0);
        if (d.p.log2s != d.p.log2s) d.mode = kDrawBad;
      }
      if (threadIdx.x == 0) {
        ds = d;
        if (part == 0) a.draw[b] = d;
      }
    }
    __syncthreads();
    const VerifyDraw d = ds;
    if (d.mode == kDrawBad) continue;
    const Tin* p = target_row<Tin>(a, b, d.pos);
    const Tin* q = d.mode == kDrawResidual ? draft_row<Tin>(a, b, d.pos) : nullptr;
    const int x = d.mode == kDrawWithout ? (int)a.ids[(int64_t)b * a.D + d.pos] : -1;
    const RowSplit sp = split_row(p, a.V);
    const int w0 = (int)((int64_t)a.cells * part / a.draw_parts);
    const int w1 = (int)((int64_t)a.cells * (part + 1) / a.draw_parts);
    for (int cell = w0 + wave; cell < w1; cell += kCellNT / 64) {
      const double s = cell_sum(a, d, d.mode, p, q, x, sp, cell);
      if ((threadIdx.x & 63) == 0) a.cell[(int64_t)b * a.cells + cell] = s;
    }
  }
}

template <typename Tin>
__global__ __launch_bounds__(kPickNT) void verify_pick(VerifyArgs a) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int NT = kPickNT;
  constexpr int NW = NT / 64;
  __shared__ double wsum[2][NW];
  __shared__ double before_s;
  __shared__ int found_s, last_s;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
    const VerifyDraw d = a.draw[b];
    int64_t* tokens = a.tokens + b * (a.D + 1);
    float* logp = a.logp + b * (a.D + 1);
    for (int i = d.pos + 1 + tid; i <= a.D; i += NT) {
      tokens[i] = -1;
      logp[i] = 0.0f;
    }
    if (tid == 0) a.accepted[b] = d.pos;
    if (d.mode == kDrawBad) {
      if (tid == 0) {
        tokens[d.pos] = -1;
        logp[d.pos] = __builtin_nanf("");
      }
      continue;
    }
    const Tin* p = target_row<Tin>(a, b, d.pos);
    const Tin* q = d.mode == kDrawResidual ? draft_row<Tin>(a, b, d.pos) : nullptr;
    const int x = d.mode == kDrawWithout ? (int)a.ids[b * a.D + d.pos] : -1;
    const RowSplit sp = split_row(p, a.V);
    double* cell = a.cell + b * a.cells;
    int mode = d.mode;
    const int run = (a.cells + NT - 1) / NT;          // cells per thread, consecutive
    const int r0 = min(tid * run, a.cells), r1 = min(r0 + run, a.cells);
    double before = 0.0, total = 0.0;                // the cells before this thread's, and all of them
    for (int attempt = 0; attempt < 2; ++attempt) {
      double own = 0.0;
      for (int c = r0; c < r1; ++c) own += cell[c];
      double incl = own;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(incl, off, 64);
        if (lane >= off) incl += o;
      }
      if (lane == 63) wsum[attempt][tid >> 6] = incl;
      if (tid == 0) {
        found_s = a.cells;
        last_s = -1;
      }
      __syncthreads();
      total = 0.0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w == tid >> 6) before = total + (incl - own);
        total += wsum[attempt][w];
      }
      if (total > 0.0) break;                        // uniform
      // p - q has no positive part: the draw is from p (the sums again, in this workgroup)
      mode = kDrawTarget;
      for (int c = tid >> 6; c < a.cells; c += NW) {
        const double s = cell_sum(a, d, mode, p, q, x, sp, c);
        if (lane == 0) cell[c] = s;
      }
      __threadfence_block();
      __syncthreads();
    }
    const double goal = (double)a.u_new[b] * total;
    int hit_cell = a.cells;
    double hit_before = before;
    {
      double c = before;
      for (int i = r0; i < r1; ++i) {
        const double w = cell[i];
        if (w > 0.0) atomicMax(&last_s, i);
        if (c + w > goal && w > 0.0) {
          atomicMin(&found_s, i);
          hit_cell = i;
          hit_before = c;
          break;
        }
        c += w;
      }
    }
    __syncthreads();
    const int found = found_s < a.cells ? found_s : last_s;   // total > 0: some weight is positive
    if (hit_cell == found) before_s = hit_before;             // one thread, if a cell was hit
    __syncthreads();
    if (tid < 64 && found >= 0) {
      double c = before_s;                                    // no cell hit: not used, c > goal fails
      if (found_s == a.cells) c = -INFINITY;
      const CellSpan s = cell_span<Tin>(sp, a.V, a.cells, found, lane);
      double w[E];
      span_weights(a, d, mode, p, q, x, s, w);
      double mine = 0.0;
#pragma unroll
      for (int j = 0; j < E; ++j) mine += w[j];
      double incl = mine;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(incl, off, 64);
        if (lane >= off) incl += o;
      }
      c += incl - mine;
      int hit = -1, last = -1;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        c += w[j];
        if (w[j] > 0.0) {
          last = s.first + j;
          if (hit < 0 && c > goal) hit = last;
        }
      }
      const uint64_t hits = __ballot(hit >= 0);
      const uint64_t lasts = __ballot(last >= 0);
      int v = -1;
      if (hits) v = __shfl(hit, __builtin_ctzll(hits), 64);
      else if (lasts) v = __shfl(last, 63 - __builtin_clzll(lasts), 64);
      if (lane == 0) {
        tokens[d.pos] = v;
        logp[d.pos] = v >= 0 ? (float)(log2_prob(a, d.p, entry_value(p, v)) * kLn2F64)
                             : __builtin_nanf("");
      }
    }
    __syncthreads();                                 // the sequence's LDS is read
  }
}

}  // namespace

int64_t verify_layout(VerifyArgs& a, int es, bool with_draft, void* workspace) {
  const int E = 16 / es;
  const int64_t chunks = a.V / E;
  const int64_t per = (int64_t)a.B * (with_draft ? 2 : 1);
  const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(per * (a.D + 1), std::max<int64_t>(per, kStatsRows)));
  // a part of two chunks per thread or more, while a launch's rows do not fill the device
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxParts, 2048 / rows, chunks / (2 * kStatsNT)}));
  a.cells = (int)((chunks + 63) / 64 + 2);
  a.draw_parts = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / std::max(a.B, 1), a.cells / 8));
  int64_t o = 0;
  auto take = [&](int64_t bytes) {
    char* p = workspace ? (char*)workspace + o : nullptr;
    o += (bytes + 15) & ~(int64_t)15;
    return p;
  };
  a.stats = (double*)take((int64_t)(a.D + 1) * a.B * 2 * a.parts * 16);
  a.cell = (double*)take((int64_t)a.B * a.cells * 8);
  a.draw = (VerifyDraw*)take((int64_t)a.B * sizeof(VerifyDraw));
  return o;
}

hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t st) {
  const unsigned g2 = (unsigned)std::min<int64_t>((int64_t)a.B * a.draw_parts, kLaunchThreads / kCellNT);
  const unsigned g3 = (unsigned)std::min<int64_t>(a.B, kLaunchThreads / kPickNT);
  // Positions in groups that fill the device; a sequence that an earlier group stops is not read on.
  // At most eight launches however many drafts there are.
  const int64_t per = (int64_t)a.B * (a.draft ? 2 : 1);
  const int group = (int)std::max<int64_t>((kStatsRows + per - 1) / per, (a.D + 1 + 7) / 8);
  for (int i0 = 0; i0 <= a.D; i0 += group) {
    const int i1 = std::min(a.D + 1, i0 + group);
    const unsigned g1 = (unsigned)std::min<int64_t>((i1 - i0) * per * a.parts, kLaunchThreads / kStatsNT);
    if (bf16) verify_stats<uint16_t><<<g1, kStatsNT, 0, st>>>(a, i0, i1);
    else verify_stats<float><<<g1, kStatsNT, 0, st>>>(a, i0, i1);
  }
  if (bf16) {
    verify_cells<uint16_t><<<g2, kCellNT, 0, st>>>(a);
    verify_pick<uint16_t><<<g3, kPickNT, 0, st>>>(a);
  } else {
    verify_cells<float><<<g2, kCellNT, 0, st>>>(a);
    verify_pick<float><<<g3, kPickNT, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace dppo
