// Verification of drafted tokens against the policy's rows (speculative decoding) with given random
// numbers: which drafts are accepted, the token drawn behind them, and the log-probs of both.
//
// Accepting compares u q(x) with p(x), and the draw finds where a running sum passes u times its
// total. Both turn on the last bits of sums over the vocabulary, and a draw from V weights goes wrong
// with a probability of about V times the running sums' error. So the draw's weights and sums are held
// in 64 bits (exponentials good to 5e-12). That costs five times a 32-bit exponential, and is spent on
// the one pair of rows that a sequence draws from:
//   1. statistics: every row's sum of exponentials with 32-bit exponentials, an error of a few 1e-6
//      that the row's size bounds. Positions come in groups; a sequence that an earlier group stops
//      is not read on.
//   2. cells: a workgroup finds where its sequence stops. An acceptance that lies within that bound is
//      decided by exact sums over its two rows. Then the weights of the row drawn from are summed over
//      cells of 64 chunks, in one pass that also sums p and q themselves: the weights max(p - q, 0) are
//      formed with the 32-bit normalisers, and the exact ones that the pass yields correct their sums
//      to first order (what changes sign within 1e-6 is second order, 1e-12).
//   3. the draw: the cell where the corrected running sum passes, then the entry, from exact weights.
//
// B = 256, D = 4, V = 151936 bf16 with drafts' logits takes 195 us in flight with other calls. Traced, one
// kernel at a time, 206 us: 118 us of statistics (positions 0 and 1: 57 us, 311 MB at 5.5 TB/s; 2 and 3:
// 40 us, 161 MB, as sequences stop; the last: 21 us, 25 MB), 76 us of cells (156 MB; bound by the 64-bit
// arithmetic, some 45 instructions per pair of entries), 12 us of the draw. One sequence (B = 1, D = 4,
// V = 32000): 5, 10 and 9 us of dependent loads and reductions.
#include "verify.h"

#include <algorithm>

#include "dppo_device.h"
#include "f64_math.h"
#include "row_split.h"

namespace dppo {

namespace {

constexpr int kStatsNT = 256;
constexpr int kCellNT = 256;
constexpr int kPickNT = 512;
constexpr int kMaxParts = 16;
// Rows of a launch of the statistics. Larger launches read more rows behind a stop, smaller ones look
// for the stops more often: 512, 1024 and 2048 take 204, 193 and 205 us at B = 256, D = 4, V = 151936 in
// bf16 with 1.9 drafts of 4 accepted, 189, 187 and 208 us with 1.2 accepted.
constexpr int64_t kStatsRows = 1024;

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
template <int E>
__device__ __forceinline__ float max_of(const float (&x)[E]) {
  if constexpr (E == 8) return max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(x[6], x[7], x[7]));
  else if constexpr (E == 4) return max3(max3(x[0], x[1], x[2]), x[3], x[3]);
  else return x[0];
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

// a / b: a 64-bit division is some 150 scalar instructions in a row, at the start of every workgroup
__device__ __forceinline__ uint64_t divide(uint64_t a, uint32_t b) {
  return a >> 32 ? a / b : (uint32_t)a / b;
}

// ------------------------------------------------------------------ where a sequence stops
// A row's sum of exponentials as the statistics have it: log2 of it, and a bound on its error. Far
// rows (logits past 2^20 log2 units, infinite ones and rows of nothing else than -inf or the type's
// lowest value among them) are left to exact arithmetic.
struct RowNorm {
  double lse2, err;
  bool far, bad;
};
enum Status { kAccept, kReject, kUnclear, kBadRow };
struct Stop {
  int pos, status;
};

// A window of a sequence's positions, for the workgroup that looks through it.
constexpr int kWindow = 16;
struct StopState {
  RowNorm norm[2][kWindow + 1];   // of the target's and the draft's rows from position `from` on
  int from;
  Stop stop;
};

// The parts of the window's rows joined: a group of lanes per row, so that their loads are in flight
// together. Called by the whole workgroup (NT threads), barriers around it are the caller's.
template <int NT>
__device__ __forceinline__ void window_norms(const VerifyArgs& a, int64_t b, int from, int n, StopState& st) {
  const int lanes = a.parts > 8 ? 16 : a.parts > 4 ? 8 : a.parts > 2 ? 4 : a.parts;
  const int part = (int)threadIdx.x % lanes;
  const int rows = min(kWindow, n - from) + 1;       // of the target; the draft has none behind the last
  for (int row = (int)threadIdx.x / lanes; row < 2 * rows; row += NT / lanes) {
    const int kind = row & 1, i = row >> 1;
    const bool in = kind == 0 || (a.draft && from + i < n);
    VerifyPart v = {-INFINITY, 0.0, -INFINITY};
    if (in && part < a.parts) v = a.stats[(((int64_t)(from + i) * a.B + b) * 2 + kind) * a.parts + part];
    double N = v.n, m = v.m;
    for (int off = 1; off < lanes; off <<= 1) {
      N = fmax(N, __shfl_xor(N, off, 64));
      m = fmax(m, __shfl_xor(m, off, 64));
    }
    double s = v.n == -INFINITY ? 0.0 : v.s * exp2_f64(v.n - N);
    for (int off = 1; off < lanes; off <<= 1) s += __shfl_xor(s, off, 64);
    if (!in || part != 0) continue;
    RowNorm r;
    r.far = !(fabs(m) * a.t2e < 1048576.0);
    r.bad = !r.far && !(s > 0.0 && s < INFINITY);
    // the sums took log2(e) / temperature in 32 bits: the logits that matter lie next to m
    r.lse2 = r.far || r.bad ? 0.0 : N + log2_f64(s) - m * ((double)(float)a.t2e - a.t2e);
    // Terms: the exponential (2^-22) and a chunk's additions (three levels, 2^-22); its argument's
    // rounding and that of log2(e) / temperature, 2^-24 ln 2 each of the log2 units below the maximum, which
    // weigh at most log2(V) <= 28 over the row. In all below 2.9e-6 of the sum.
    r.err = 4e-6;
    st.norm[kind][i] = r;
  }
}

// The first of the drafts [from, n) of sequence b that is not clearly accepted (position n if there is
// none) and its status, by the whole workgroup. With `write`, the accepted drafts and their log-probs
// go to the outputs. Rows behind that draft may have statistics that were never computed; they decide
// nothing. Afterwards st.norm holds the position's rows, at st.stop.pos - st.from.
template <typename Tin, int NT>
__device__ __forceinline__ Stop first_stop(const VerifyArgs& a, int b, int from, int n, bool write, StopState& st) {
  for (;; from += kWindow) {
    // a draft per lane; what its decision reads is in flight together with the statistics
    const int lane = threadIdx.x;
    const int i = from + lane;
    const bool in = lane < kWindow && i < n;
    int64_t x = -1;
    float u = 0.0f, zp = 0.0f, zq = 0.0f;
    if (in) {
      x = a.ids[(int64_t)b * a.D + i];
      u = a.u[(int64_t)b * a.D + i];
      if (x >= 0 && x < a.V) {
        zp = entry_value(target_row<Tin>(a, b, i), x);
        if (a.draft) zq = entry_value(draft_row<Tin>(a, b, i), x);
      }
    }
    __syncthreads();                                 // st is read
    window_norms<NT>(a, b, from, n, st);
    __syncthreads();
    if (threadIdx.x < 64) {
      int status = kAccept;
      float out = 0.0f;
      if (in) {
        const RowNorm p = st.norm[0][lane];
        RowNorm q{};
        if (a.draft) q = st.norm[1][lane];
        if (x < 0 || x >= a.V || p.bad || q.bad) {
          status = kBadRow;
        } else if (p.far || q.far) {
          status = kUnclear;
        } else {
          const double lp = __builtin_fma((double)zp, a.t2e, -p.lse2);
          const double q_x = a.draft ? exp2_f64(__builtin_fma((double)zq, a.t2e, -q.lse2)) : 1.0;
          const double uq = (double)u * q_x, pp = exp2_f64(lp);
          const double mu = 1.0 + (p.err + q.err);
          status = uq * mu < pp ? kAccept : (uq < pp * mu ? kUnclear : kReject);
          if (pp == 0.0) status = kReject;
          out = (float)(lp * kLn2F64);
        }
      }
      const uint64_t stops = __ballot(status != kAccept);
      const int first = stops ? __builtin_ctzll(stops) : 64;
      if (write && in && lane < first) {
        a.tokens[(int64_t)b * (a.D + 1) + i] = x;
        a.logp[(int64_t)b * (a.D + 1) + i] = out;
      }
      status = __shfl(status, first & 63, 64);
      if (lane == 0) {
        st.from = from;
        st.stop = stops ? Stop{from + first, status} : Stop{min(from + kWindow, n), kAccept};
      }
    }
    __syncthreads();
    const Stop s = st.stop;
    if (s.status != kAccept || s.pos == n) return s;
  }
}

// ------------------------------------------------------------------ statistics
// One part of one row per workgroup, for the positions [i0, i1); positions outermost. Sequences that
// clearly stop before i0 (whose statistics are complete: earlier launches) are skipped.
template <typename Tin>
__global__ __launch_bounds__(kStatsNT, 4) void verify_stats(VerifyArgs a, int i0, int i1) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int NT = kStatsNT;
  constexpr int U = 8;
  constexpr int NW = NT / 64;
  __shared__ double red[3 * NW];
  __shared__ StopState st;
  const int tid = threadIdx.x;
  const int kinds = a.draft ? 2 : 1;
  const float L = (float)a.t2e;
  const int64_t items = (int64_t)(i1 - i0) * a.B * kinds * a.parts;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint64_t row = divide(item, a.parts);
    const int part = (int)(item - row * a.parts);
    const uint64_t pos_b = kinds == 2 ? row >> 1 : row;
    const int kind = kinds == 2 ? (int)(row & 1) : 0;
    const uint64_t pos = divide(pos_b, a.B);
    const int b = (int)(pos_b - pos * a.B);
    const int i = i0 + (int)pos;
    if (i + kind > drafts_of(a, b)) continue;        // uniform: not a row of this sequence
    const Tin* z = kind ? draft_row<Tin>(a, b, i) : target_row<Tin>(a, b, i);
    const RowSplit sp = split_row(z, a.V);
    const int c0 = (int)((int64_t)sp.nfull * part / a.parts);
    const int n = (int)((int64_t)sp.nfull * (part + 1) / a.parts) - c0;
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead + (int64_t)c0 * E, n * 16);
    if (i0 > 0) {
      const int s = first_stop<Tin, NT>(a, b, 0, i0, false, st).status;
      if (s == kReject || s == kBadRow) continue;
    }
    uint32_t r[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) load16<kAuxLast>(r[u], rz, tid * 16, u * NT * 16);
    float N = kNoShift, m = -INFINITY;               // 2^N s so far; the largest logit
    double s = 0.0;
    auto add = [&](const auto& x) {
      const float cm = max_of(x);
      add_logits(N, s, x, cm, L);
      m = fmaxf(m, cm);
    };
    if (part == 0 && tid < sp.nedge) {
      const float x[1] = {entry_value(z, sp.template entry<E>(tid))};
      add(x);
    }
    for (int base = 0; base < n; base += U * NT) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (base + u * NT >= n) break;               // uniform
        float x[E];
        unpack<Tin>(r[u], x);
        if (base + (U + u) * NT < n) load16<kAuxLast>(r[u], rz, tid * 16, (base + (U + u) * NT) * 16);
        if (tid < n - base - u * NT) add(x);
      }
    }
    // the wave's largest shift, then one exact scale per thread
    const float M = wave_max(N);
    s = wave_sum_f64(N == M ? s : s * (double)exp2_hw(N - M));
    m = wave_max(m);
    __syncthreads();                                 // the last item's partials are read
    if ((tid & 63) == 0) {
      red[tid >> 6] = shift_of(M);
      red[NW + (tid >> 6)] = s;
      red[2 * NW + (tid >> 6)] = m;
    }
    __syncthreads();
    if (tid == 0) {
      VerifyPart o = {red[0], 0.0, red[2 * NW]};
      for (int w = 1; w < NW; ++w) {
        o.n = fmax(o.n, red[w]);
        o.m = fmax(o.m, red[2 * NW + w]);
      }
      for (int w = 0; w < NW; ++w) o.s += red[w] == o.n ? red[NW + w] : red[NW + w] * exp2_f64(red[w] - o.n);
      a.stats[(((int64_t)i * a.B + b) * 2 + kind) * a.parts + part] = o;
    }
  }
}

// ------------------------------------------------------------------ exact rows (rare)
// log2 of an entry's probability under an exact normaliser.
__device__ __forceinline__ double log2_prob(const VerifyArgs& a, const VerifyNorm& n, float z) {
  return __builtin_fma((double)z - n.m, a.t2e, -n.log2s);
}

// A row's exact normaliser, by the workgroup; log2s is NaN for a row holding NaN or +inf, or only -inf.
template <typename Tin, int NT>
__device__ VerifyNorm exact_norm(const VerifyArgs& a, const Tin* z, double* red) {
  constexpr int NW = NT / 64;
  float m = -INFINITY;
  for (int e = threadIdx.x; e < a.V; e += NT) m = fmaxf(m, entry_value(z, e));
  m = wave_max(m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  double M = red[0];
  for (int w = 1; w < NW; ++w) M = fmax(M, red[w]);
  double s = 0.0;
  if (M != -INFINITY)
    for (int e = threadIdx.x; e < a.V; e += NT) s += exp2_f64(((double)entry_value(z, e) - M) * a.t2e);
  s = wave_sum_f64(s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < NW; ++w) s += red[w];
  __syncthreads();
  return {M, s > 0.0 && s < INFINITY ? log2_f64(s) : (double)__builtin_nanf("")};
}

// ------------------------------------------------------------------ weights
// p and q of E logits each, as scaled (VerifyDraw); entries below 2^-1000 of p's or q's scale are
// held there, and flushed where that could show.
constexpr double kFlush = 1e-280;
__device__ __forceinline__ float lowest_logit(const VerifyArgs& a, double s) {
  return (float)((-s / kExpTable - 1000.0) / a.t2e);
}
template <int E>
__device__ __forceinline__ void probs(const VerifyArgs& a, const VerifyDraw& d, double s, const VerifyNorm& n,
                                      const float (&z)[E], const double* table, double (&w)[E]) {
  if (d.far) {
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = exp2_f64(log2_prob(a, n, z[j]));
  } else {
    const double K = a.t2e * kExpTable, sm = s + kRoundMagic;
    const float low = lowest_logit(a, s);
#pragma unroll
    for (int j = 0; j < E; ++j)
      w[j] = exp2_tab((double)__builtin_elementwise_maximum(z[j], low), K, sm, table);
  }
}

// exact_norm of a row whose log2 sum is about lse2 and not large, from weights as above, in a sixth of its
// time: a decision at its border costs 85 us instead of 540 (V = 151936 bf16). A chance of some 1e-5 each.
template <typename Tin, int NT>
__device__ VerifyNorm near_norm(const VerifyArgs& a, const Tin* z, double lse2, const double* table, double* red) {
  constexpr int NW = NT / 64;
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int U = 2;
  const int tid = threadIdx.x;
  const double shift = -__builtin_rint(lse2 * kExpTable), K = a.t2e * kExpTable, sm = shift + kRoundMagic;
  const float low = lowest_logit(a, shift);
  const RowSplit sp = split_row(z, a.V);
  const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead, sp.nfull * 16);
  double s = 0.0;
  auto add = [&](float x) { s += exp2_tab((double)__builtin_elementwise_maximum(x, low), K, sm, table); };
  if (tid < sp.nedge) add(entry_value(z, sp.template entry<E>(tid)));
#pragma unroll 1
  for (int c = tid; c < sp.nfull; c += U * NT) {
    uint32_t r[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) load16<kAuxLast>(r[u], rz, c * 16, u * NT * 16);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c + u * NT >= sp.nfull) break;
      float x[E];
      unpack<Tin>(r[u], x);
#pragma unroll
      for (int j = 0; j < E; ++j) add(x[j]);
    }
  }
  s = wave_sum_f64(s);
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < NW; ++w) s += red[w];
  __syncthreads();
  return {0.0, s > 0.0 && s < INFINITY ? log2_f64(s) - shift / kExpTable : (double)__builtin_nanf("")};
}

// Cell 0 holds the entries before the target row's whole chunks, cell c the 64 chunks from 64 (c - 1)
// on, the last cell the entries behind them. A lane's entries of a cell: `count` of them (a chunk or a
// single one) from `first` on.
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
// Its logits in `row`, -inf past the span. chunks: the span's start is 16-byte aligned in this row.
template <typename Tin>
__device__ __forceinline__ void span_logits(const Tin* row, const CellSpan& s, bool chunks, float (&z)[16 / sizeof(Tin)]) {
  constexpr int E = 16 / (int)sizeof(Tin);
  if (s.count == E && chunks) {
    unpack<Tin>(*(const u32x4*)(row + s.first), z);
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j) z[j] = j < s.count ? entry_value(row, s.first + j) : -INFINITY;
  }
}

// 16 bytes of a row at any alignment, in a load of their own size
typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
template <typename Tin>
__device__ __forceinline__ Words all_lowest() {
  const uint32_t w = sizeof(Tin) == 2 ? 0xFF80FF80u : 0xFF800000u;   // -inf
  return Words{w, w, w, w};
}
template <typename Tin>
__device__ __forceinline__ void set_first(Words& w, Tin v) {
  if constexpr (sizeof(Tin) == 2) w[0] = 0xFF800000u | v;
  else w[0] = __float_as_uint(v);
}

// A row drawn from, and the workgroup's handle on it.
template <typename Tin>
struct DrawRows {
  const Tin *p, *q;
  bool q_chunks;         // q's rows have p's offset within 16 bytes
  int x;                 // the drafted token that p is drawn without, or -1
  RowSplit split;
};
template <typename Tin>
__device__ __forceinline__ DrawRows<Tin> draw_rows(const VerifyArgs& a, const VerifyDraw& d, int64_t b) {
  DrawRows<Tin> r;
  r.p = target_row<Tin>(a, b, d.pos);
  r.q = d.mode == kDrawResidual ? draft_row<Tin>(a, b, d.pos) : nullptr;
  r.q_chunks = (((uintptr_t)r.p - (uintptr_t)r.q) & 15) == 0;
  r.x = d.mode == kDrawWithout ? (int)a.ids[b * a.D + d.pos] : -1;
  r.split = split_row(r.p, a.V);
  return r;
}

// ------------------------------------------------------------------ cells
// 128 registers: at 96 (five waves per SIMD) it spills, and 199 us become 214 (B = 256, D = 4, V = 151936).
template <typename Tin>
__global__ __launch_bounds__(kCellNT, 4) void verify_cells(VerifyArgs a) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int NW = kCellNT / 64;
  __shared__ double table[kExpTable];
  __shared__ double red[NW];
  __shared__ StopState st;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  exp2_table_fill(table);
  for (int64_t item = blockIdx.x; item < (int64_t)a.B * a.draw_parts; item += gridDim.x) {
    const int b = (int)divide(item, a.draw_parts);
    const int part = (int)(item - (int64_t)b * a.draw_parts);
    const int n = drafts_of(a, b);
    // where the sequence stops; every workgroup of a sequence comes to the same answer
    VerifyDraw d{};
    for (int from = 0;;) {
      const Stop s = first_stop<Tin, kCellNT>(a, b, from, n, part == 0, st);
      d.pos = s.pos;
      d.mode = s.status == kBadRow ? kDrawBad
               : s.pos == n        ? kDrawTarget
                                   : (a.draft ? kDrawResidual : kDrawWithout);
      if (s.status != kUnclear) break;
      // within the statistics' error, or beyond their range: from exact sums over the two rows
      const int64_t x = a.ids[(int64_t)b * a.D + s.pos];
      const Tin* p = target_row<Tin>(a, b, s.pos);
      // (log2s alone holds 2^-40 of a probability where it is below 4096)
      auto norm_of = [&](const Tin* z, const RowNorm& n) {
        return !n.far && fabs(n.lse2) < 4096.0 ? near_norm<Tin, kCellNT>(a, z, n.lse2, table, red)
                                               : exact_norm<Tin, kCellNT>(a, z, red);
      };
      d.p = norm_of(p, st.norm[0][s.pos - st.from]);
      d.q = {0.0, 0.0};
      double q = 1.0;
      if (a.draft) {
        const Tin* qr = draft_row<Tin>(a, b, s.pos);
        d.q = norm_of(qr, st.norm[1][s.pos - st.from]);
        q = exp2_f64(log2_prob(a, d.q, entry_value(qr, x)));
      }
      const double lp = log2_prob(a, d.p, entry_value(p, x));
      if (d.p.log2s != d.p.log2s || d.q.log2s != d.q.log2s) {
        d.mode = kDrawBad;
        break;
      }
      if (!((double)a.u[(int64_t)b * a.D + s.pos] * q < exp2_f64(lp))) break;
      if (part == 0 && tid == 0) {
        a.tokens[(int64_t)b * (a.D + 1) + s.pos] = x;
        a.logp[(int64_t)b * (a.D + 1) + s.pos] = (float)(lp * kLn2F64);
      }
      from = s.pos + 1;
    }
    if (d.mode != kDrawBad) {
      const RowNorm p = st.norm[0][d.pos - st.from];
      RowNorm q{};
      if (d.mode == kDrawResidual) q = st.norm[1][d.pos - st.from];
      d.far = __builtin_amdgcn_readfirstlane(p.far || q.far);
      if (p.bad || q.bad) d.mode = kDrawBad;
      if (d.far && d.mode != kDrawBad) {             // uniform
        d.p = exact_norm<Tin, kCellNT>(a, target_row<Tin>(a, b, d.pos), red);
        if (d.mode == kDrawResidual) d.q = exact_norm<Tin, kCellNT>(a, draft_row<Tin>(a, b, d.pos), red);
        else d.q = {0.0, 0.0};
        if (d.p.log2s != d.p.log2s || d.q.log2s != d.q.log2s) d.mode = kDrawBad;
      }
      d.sp = -__builtin_rint(p.lse2 * kExpTable);
      d.sq = -__builtin_rint(q.lse2 * kExpTable);
      d.phi = d.far ? 1.0
                    : exp2_f64(((-d.sq / kExpTable) - q.lse2) - ((-d.sp / kExpTable) - p.lse2));
    }
    if (part == 0 && tid == 0) a.draw[b] = d;
    if (d.mode == kDrawBad) continue;                // uniform
    const DrawRows<Tin> rows = draw_rows<Tin>(a, d, b);
    const int w0 = (int)((int64_t)a.cells * part / a.draw_parts);
    const int w1 = (int)((int64_t)a.cells * (part + 1) / a.draw_parts);
    // The next cell's logits are read ahead, as they are; q's in p's chunks, whatever their alignment.
    const Words low = all_lowest<Tin>();
    Words wp, wq;
    auto fetch = [&](int cell) {
      const CellSpan s = cell < w1 ? cell_span<Tin>(rows.split, a.V, a.cells, cell, lane) : CellSpan{0, 0};
      // uniform; a row of fewer entries than fill a chunk at its offset has none
      if (cell > 0 && cell < a.cells - 1 && rows.split.nfull > 0) {
        // lanes past the chunks read the last one
        const int e = rows.split.lead + (min((cell - 1) * 64 + lane, rows.split.nfull - 1)) * E;
        wp = *(const u32x4*)(rows.p + e);
        if (d.mode == kDrawResidual) wq = *(const Words*)(rows.q + e);
      } else {
        wp = wq = low;
        if (s.count) {
          set_first<Tin>(wp, rows.p[s.first]);
          if (d.mode == kDrawResidual) set_first<Tin>(wq, rows.q[s.first]);
        }
      }
      return s;
    };
    CellSpan s = {0, 0};
    if (w0 + wave < w1) s = fetch(w0 + wave);
    for (int cell = w0 + wave; cell < w1; cell += NW) {
      const CellSpan now = s;
      float cp[E], cq[E];
      unpack<Tin>(now.count ? wp : low, cp);
      unpack<Tin>(now.count ? wq : low, cq);
      if (cell + NW < w1) s = fetch(cell + NW);
      VerifyCell c = {0.0, 0.0, 0.0, 0.0};
      double w[E];
      probs(a, d, d.sp, d.p, cp, table, w);
#pragma unroll
      for (int j = 0; j < E; ++j) c.p += w[j];
      if (d.mode == kDrawResidual) {
        double v[E];
        probs(a, d, d.sq, d.q, cq, table, v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          c.q += v[j];
          const double r = __builtin_fma(-d.phi, v[j], w[j]);
          c.r += r > kFlush ? r : 0.0;
          c.slope += r > kFlush ? v[j] : 0.0;
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) c.r += now.first + j == rows.x ? 0.0 : w[j];
      }
      const double sum = wave_sum4_f64({c.r > kFlush ? c.r : 0.0, c.slope, c.p > kFlush ? c.p : 0.0, c.q});
      if (lane < 4) ((double*)(a.cell + (int64_t)b * a.cells + cell))[lane] = sum;
    }
  }
}

// ------------------------------------------------------------------ the draw
template <typename Tin>
__global__ __launch_bounds__(kPickNT, 4) void verify_pick(VerifyArgs a) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int NT = kPickNT;
  constexpr int NW = NT / 64;
  __shared__ double table[kExpTable];
  __shared__ double wsum[3][NW];
  __shared__ double before_s;
  __shared__ int found_s, last_s;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  exp2_table_fill(table);
  for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
    // this thread's cells (consecutive), the first of them in registers, in flight together with the rest
    // (all of them up to V = 2^20 bf16, 2^19 fp32)
    constexpr int R = 4;
    const VerifyCell* cells = a.cell + b * a.cells;
    const int run = (a.cells + NT - 1) / NT;
    const int r0 = min(tid * run, a.cells), r1 = min(r0 + run, a.cells);
    VerifyCell own_cells[R];
#pragma unroll
    for (int k = 0; k < R; ++k) own_cells[k] = r0 + k < r1 ? cells[r0 + k] : VerifyCell{0.0, 0.0, 0.0, 0.0};
    const double u_new = a.u_new[b];
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
    // f(cell, its sums) over this thread's cells, until it returns true
    auto each = [&](auto&& f) {
      bool done = false;
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (!done && r0 + k < r1) done = f(r0 + k, own_cells[k]);
      for (int c = r0 + R; c < r1 && !done; ++c) done = f(c, cells[c]);
    };
    // p's and q's exact totals: the scale that q has to have against p
    double tp = 0.0, tq = 0.0;
    each([&](int, const VerifyCell& c) {
      tp += c.p;
      tq += c.q;
      return false;
    });
    tp = wave_sum_f64(tp);
    tq = wave_sum_f64(tq);
    if (lane == 0) {
      wsum[0][wave] = tp;
      wsum[1][wave] = tq;
    }
    if (tid == 0) {
      found_s = a.cells;
      last_s = -1;
    }
    __syncthreads();
    tp = tq = 0.0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      tp += wsum[0][w];
      tq += wsum[1][w];
    }
    bool residual = d.mode == kDrawResidual;
    const double scale = residual ? tp / tq : 0.0;   // of q; phi is the scale the cells used
    bool from_p = d.mode == kDrawTarget;
    auto weight = [&](const VerifyCell& c) {
      if (from_p) return c.p;
      return residual ? fmax(c.r - (scale - d.phi) * c.slope, 0.0) : c.r;
    };
    double before = 0.0, total = 0.0, own = 0.0;     // the cells before this thread's, all, its own
    for (;;) {
      own = 0.0;
      each([&](int, const VerifyCell& c) {
        own += weight(c);
        return false;
      });
      double incl = own;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(incl, off, 64);
        if (lane >= off) incl += o;
      }
      if (lane == 63) wsum[2][wave] = incl;
      __syncthreads();
      total = 0.0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w == wave) before = total + (incl - own);
        total += wsum[2][w];
      }
      // p - q without a positive part beyond rounding (p = q): the draw is from p
      if (from_p || total > 1e-12 * tp) break;       // uniform
      from_p = true;
      residual = false;
      __syncthreads();
    }
    const double goal = u_new * total;
    int hit_cell = a.cells;
    double hit_before = before;
    {
      double sum = before;
      each([&](int i, const VerifyCell& c) {
        const double w = weight(c);
        if (w > 0.0) atomicMax(&last_s, i);
        if (sum + w > goal && w > 0.0) {
          atomicMin(&found_s, i);
          hit_cell = i;
          hit_before = sum;
          return true;
        }
        sum += w;
        return false;
      });
    }
    __syncthreads();
    const int found = found_s < a.cells ? found_s : last_s;   // total > 0: some weight is positive
    if (hit_cell == found) before_s = hit_before;
    __syncthreads();
    if (tid < 64 && found >= 0) {
      const DrawRows<Tin> rows = draw_rows<Tin>(a, d, b);
      // No cell passed the goal (rounding, or u = 1): the last positive weight. A cell whose weight is
      // rounding alone (u = 0 finds it) has no entry: the next entry behind it, or else the last before it.
      const bool passed = found_s < a.cells;
      int v = -1;
      float zv = 0.0f;
#pragma unroll 1
      for (int cell = found, way = 0;;) {
        const CellSpan s = cell_span<Tin>(rows.split, a.V, a.cells, cell, lane);
        float z[E];
        double w[E];
        span_logits(rows.p, s, true, z);
        probs(a, d, d.sp, d.p, z, table, w);
        if (residual) {
          double v[E];
          float y[E];
          span_logits(rows.q, s, rows.q_chunks, y);
          probs(a, d, d.sq, d.q, y, table, v);
#pragma unroll
          for (int j = 0; j < E; ++j) w[j] = __builtin_fma(-scale, v[j], w[j]);
        }
        double mine = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
          if (!(w[j] > kFlush) || (!from_p && s.first + j == rows.x)) w[j] = 0.0;
          mine += w[j];
        }
        double incl = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const double o = __shfl_up(incl, off, 64);
          if (lane >= off) incl += o;
        }
        double c = (way > 0 ? INFINITY : way == 0 && passed ? before_s : -INFINITY) + (incl - mine);
        int hit = -1, last = -1;
        float z_hit = 0.0f, z_last = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
          c += w[j];
          if (w[j] > 0.0) {
            last = s.first + j;
            z_last = z[j];
            if (hit < 0 && c > goal) {
              hit = last;
              z_hit = z[j];
            }
          }
        }
        const uint64_t hits = __ballot(hit >= 0);
        const uint64_t lasts = __ballot(last >= 0);
        if (hits) {
          const int from = __builtin_ctzll(hits);
          v = __shfl(hit, from, 64);
          zv = __shfl(z_hit, from, 64);
        } else if (lasts) {
          const int from = 63 - __builtin_clzll(lasts);
          v = __shfl(last, from, 64);
          zv = __shfl(z_last, from, 64);
        }
        if (v >= 0) break;
        if (way >= 0 && passed && cell + 1 < a.cells) {
          way = 1;
          ++cell;
        } else {
          if (way > 0) cell = found;
          way = -1;
          if (--cell < 0) break;
        }
      }
      if (lane == 0) {
        tokens[d.pos] = v;
        float out = __builtin_nanf("");
        if (v >= 0) {
          const double l = d.far ? log2_prob(a, d.p, zv)
                                 : __builtin_fma((double)zv, a.t2e, d.sp / kExpTable) - log2_f64(tp);
          out = (float)(l * kLn2F64);
        }
        logp[d.pos] = out;
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
  // A part of two chunks per thread or more, while a launch's rows do not fill the device: 2048, 4096
  // and 6144 workgroups take 107, 96 and 99 us at B = 128, D = 8, V = 100000 in bf16, 45, 45 and 49 us at
  // B = 32, D = 5, V = 151936.
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxParts, 4096 / rows, chunks / (2 * kStatsNT)}));
  a.cells = (int)((chunks + 63) / 64 + 2);
  // Every workgroup of the weights first finds where its sequence stops. 512, 1024 and 2048 of them: 211,
  // 198 and 201 us at B = 256, D = 4, V = 151936 in bf16, 49, 48 and 52 us at B = 64, V = 50257 in fp32.
  a.draw_parts = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / std::max(a.B, 1), a.cells / 8));
  int64_t o = 0;
  auto take = [&](int64_t bytes) {
    char* p = workspace ? (char*)workspace + o : nullptr;
    o += (bytes + 15) & ~(int64_t)15;
    return p;
  };
  a.stats = (VerifyPart*)take((int64_t)(a.D + 1) * a.B * 2 * a.parts * sizeof(VerifyPart));
  a.cell = (VerifyCell*)take((int64_t)a.B * a.cells * sizeof(VerifyCell));
  a.draw = (VerifyDraw*)take((int64_t)a.B * sizeof(VerifyDraw));
  return o;
}

hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t st) {
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
  const unsigned g2 = (unsigned)std::min<int64_t>((int64_t)a.B * a.draw_parts, kLaunchThreads / kCellNT);
  const unsigned g3 = (unsigned)std::min<int64_t>(a.B, kLaunchThreads / kPickNT);
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
