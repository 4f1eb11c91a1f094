// Distillation from a teacher's top logits: per row the divergence between the teacher's record (k
// values with their token ids) and the student's softmax, and its gradient, with the logits read
// once and dlogits written once.
//
// With q = softmax(z / tau), p the record's probabilities, P = sum p, Q = sum of q over the record's
// tokens:
//   renormalised record: l = sum p_k (log p_k - log q_k),              f = g = P
//   with the tail:       l + Pt log(Pt / Qt), Pt = 1 - P, Qt = 1 - Q,  f = P - Pt Q / Qt, g = P + Pt
//   dz_v = s / tau * f q_v outside the record, s / tau * (g q_v - p_v) inside it.
// Qt is summed over the entries outside the record: 1 - Q would lose it where the student is nearly
// sure of the record's tokens. So the record's entries leave the sum of exponentials when their
// chunk is read, and the record's own exponentials join it afterwards.
//
// A workgroup handles a row (some shapes loop over rows). The row's first NT NC 16-byte chunks
// stay in registers as they were read, the next KS NT in LDS, and only the rest of a longer row is
// read again for the gradient. Every entry belongs to one thread (RowSplit; chunk c to thread
// c mod NT), which finds the record's tokens among its entries in a list of its own (built in LDS by
// the threads that hold the record); a bit per chunk slot tells it which chunks to look at. The
// record's own arithmetic runs in 64 bits on one wave: k is small, and the loss is a difference of
// log-probabilities.
//
// Bound by HBM, with the record's arithmetic in the middle of every row: T = 8192, V = 151936 bf16, k = 64
// takes 1038 us (4.8 TB/s, logits read and dlogits written once; a device copy of 4 GiB ran at 4.75 TB/s),
// T = 4096, V = 50257 fp32, k = 128 404 us (4.1 TB/s, one row per compute unit at a time), T = 4096, V =
// 32000 bf16, k = 32 with 40 % of the rows masked 94 us. T = 256, V = 1024: 11 us, a row's chain of steps.
#include "distill.h"

#include <algorithm>
#include <mutex>

#include "dppo_device.h"
#include "f64_math.h"
#include "row_common.h"
#include "row_split.h"

namespace dppo {

namespace {

constexpr int kMaxK = DPPO_MAX_TOP;
// Least tail mass a student is given: the tail's gradient carries 1 / Qt. Below it the gradient's formulas
// go on with the floor, though the loss's tail term is constant there: its slope would drop the pull
// towards the tail at once.
constexpr double kTailFloor = 5.9604644775390625e-08;   // 2^-24

// A row's record in LDS. Two of them alternate between the rows that are evaluated: threads still
// in one row's gradient read its record while others prepare the next row's.
template <int NT>
struct Record {
  int head[NT];        // first record entry in a thread's list, -1: none; reset by its thread
  int16_t next[kMaxK];
  int id[kMaxK];
  float grad[kMaxK];   // dlogits at the entry's token
  uint8_t again[kMaxK];  // the token stands at a lower place of the record too
};

struct RecordMath {    // one row at a time, between two barriers
  float value[kMaxK];  // the record's values, then its probabilities p
  float z[kMaxK];      // the student's logits, then its probabilities q
  int any_again;
  float w, lse2;
  int far;             // the row's sum in 32 bits says nothing (kFarLog2)
};

// The record's part of a row, by one wave: lane holds entries lane, lane + 64, ... N, S: the sum of
// exponentials outside the record (2^N S, in log2 units). Everything an entry needs waits in LDS and
// the loops are not unrolled, and what all lanes share sits in scalar registers: next to a row in
// vector registers there is no room for more.
template <class Rec>
__device__ __forceinline__ void record_math(const DistillArgs& a, int64_t row, float scale, float N, float S,
                                            Rec& rec, RecordMath& m) {
  const int lane = threadIdx.x & 63;
  const int k = a.k;
  const double zl = (double)a.l2e;
  // -inf marks an empty entry here: its probability and its term are 0 either way
  double tm = -INFINITY, zm = N;
#pragma unroll 1
  for (int j = lane; j < k; j += 64) {
    tm = fmax(tm, (double)m.value[j] * a.t2e);
    zm = fmax(zm, (double)m.z[j] * zl);
  }
  zm = wave_uniform(wave_max_f64(zm));
  tm = wave_uniform(wave_max_f64(tm));
  const double zs = zm == -INFINITY ? 0.0 : zm;
  // the sums of exponentials around the maxima
  double st = 0.0, sq = 0.0;
#pragma unroll 1
  for (int j = lane; j < k; j += 64) {
    const double tj = (double)m.value[j] * a.t2e;
    if (tj != -INFINITY) st += exp2_f64(tj - tm);
    if (!rec.again[j]) sq += exp2_f64((double)m.z[j] * zl - zs);
  }
  sq = wave_uniform(wave_sum_f64(sq));
  double c;
  if (a.tlse) {
    c = (double)uload(a.tlse + row) * kLog2eF64;
  } else {
    st = wave_uniform(wave_sum_f64(st));
    c = st == 0.0 ? 0.0 : wave_uniform(tm + log2_f64(st));   // 0: an empty record, or one of -inf alone
  }
  const double rest = wave_uniform(N == -INFINITY ? 0.0 : (double)S * exp2_f64((double)N - zs));
  const double total = sq + rest;
  const double lse2 = zm == -INFINITY ? (double)__builtin_nanf("") : wave_uniform(zs + log2_f64(total));
  double l = 0.0, P = 0.0, Q = 0.0;
#pragma unroll 1
  for (int j = lane; j < k; j += 64) {
    const double tj = (double)m.value[j] * a.t2e;
    const double lq = (double)m.z[j] * zl - lse2;
    const double p = tj == -INFINITY ? 0.0 : exp2_f64(tj - c);
    const double q = rec.id[j] < 0 ? 0.0 : exp2_f64(lq);
    if (p != 0.0) l += p * ((tj - c) - lq) * kLn2F64;
    P += p;
    if (!rec.again[j]) Q += q;
    m.value[j] = (float)p;                 // the gradient g q - p is held in 32 bits
    m.z[j] = (float)q;
  }
  l = wave_uniform(wave_sum_f64(l));
  P = wave_uniform(wave_sum_f64(P));
  double f = P, g = P;
  if (a.tlse) {
    Q = wave_uniform(wave_sum_f64(Q));
    const double Pt = 1.0 - P > 0.0 ? 1.0 - P : 0.0;
    const double out = rest / total;       // NaN for a row of no softmax, which has to stay one
    const double Qt = out < kTailFloor ? kTailFloor : out;
    if (Pt > 0.0) l += Pt * log2_f64(Pt / Qt) * kLn2F64;
    f = P - Pt * Q / Qt;
    g = P + Pt;
  }
  const double s = (double)scale * a.inv_tau;
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll 1
  for (int j = lane; j < k; j += 64) {
    double p = m.value[j];
    if (m.any_again)
      for (int i = j + 1; i < k; ++i)
        if (rec.id[i] == rec.id[j]) p += m.value[i];
    rec.grad[j] = (float)(s * (g * m.z[j] - p));
  }
  if (lane == 0) {
    // what rounding lse2 to 32 bits leaves over goes into the factor
    const float l2 = (float)lse2;
    m.lse2 = l2;
    // zm is the row's maximum; entries outside the record that lie far below it weigh nothing
    m.far = !(S < INFINITY) || !(fabs(zm) < (double)kFarLog2);
    m.w = (float)(s * f * exp2_f64((double)l2 - lse2));
    a.loss_tok[row] = (float)l;
  }
}

template <typename Tin>
__device__ __forceinline__ float entry_value(const Tin* p, int64_t i) {
  if constexpr (sizeof(Tin) == 2) return bf16_to_f32(p[i]);
  else return p[i];
}

// A far row (kFarLog2), from its logits in memory: their differences to the row's maximum take their place
// (both give the same softmax), in 64 bits in the sum. A row holding NaN or +inf, or only -inf, keeps
// its logits and comes out NaN. By the whole workgroup, once its other rows are done; thread tid has the entries
// tid, tid + NT, ...; red holds a double per wave.
constexpr uint8_t kFlagFar = 0x80;       // in flags_out until the row's turn comes
template <typename Tin, int NT>
__device__ __forceinline__ void far_row(const DistillArgs& a, int64_t row, float scale, Record<NT>& rec, RecordMath& m,
                                     double* red) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x;
  const Tin* z = (const Tin*)a.logits + row * a.ld;
  Tin* d = a.dlogits ? (Tin*)a.dlogits + row * a.ldd : nullptr;
  const int V = a.V;
  __syncthreads();                         // the last row's LDS is free
  rec.head[tid] = -1;
  if (tid == 0) m.any_again = 0;
  __syncthreads();
  for (int j = tid; j < a.k; j += NT) {
    const int id = a.tokens[row * a.k + j];
    rec.id[j] = id;
    rec.again[j] = 0;
    m.value[j] = id < 0 ? -INFINITY : a.values[row * a.k + j];
    if (id >= 0) rec.next[j] = (int16_t)atomicExch(&rec.head[id % NT], j);
  }
  float base = -INFINITY;
  for (int e = tid; e < V; e += NT) {
    const float x = entry_value(z, e);
    base = x != x ? INFINITY : fmaxf(base, x);
  }
  base = wave_max(base);
  if ((tid & 63) == 0) red[tid >> 6] = base;
  __syncthreads();
  for (int w = 0; w < NW; ++w) base = fmaxf(base, (float)red[w]);
  if (!(fabsf(base) < INFINITY)) base = 0.0f;
  const int head = rec.head[tid];
  for (int j = head; j >= 0; j = rec.next[j])
    for (int j2 = rec.next[j]; j2 >= 0; j2 = rec.next[j2])
      if (rec.id[j2] == rec.id[j]) {
        rec.again[j > j2 ? j : j2] = 1;
        m.any_again = 1;
      }
  auto place = [&](int e) {                // of an entry in the record, -1: none
    int at = -1;
    for (int j = head; j >= 0; j = rec.next[j])
      if (rec.id[j] == e && !rec.again[j]) at = j;
    return at;
  };
  double s = 0.0;
  for (int e = tid; e < V; e += NT)
    if (place(e) < 0) s += exp2_f64((double)(entry_value(z, e) - base) * (double)a.l2e);
  s = wave_sum_f64(s);
  for (int j = tid; j < a.k; j += NT) m.z[j] = rec.id[j] < 0 ? -INFINITY : entry_value(z, rec.id[j]) - base;
  __syncthreads();                         // red is read
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < NW; ++w) s += red[w];
  if (tid < 64) record_math(a, row, scale * (a.tscale ? uload(a.tscale + row) : 1.0f), 0.0f, (float)s, rec, m);
  if (tid == 0) a.flags[row] = (uint8_t)DPPO_FLAG_VALID;
  __syncthreads();
  if (!d) return;
  const float w = m.w, l2 = m.lse2;
  for (int e = tid; e < V; e += NT) {
    const int j = place(e);
    const float o = j >= 0 ? rec.grad[j] : w * exp2_hw(__builtin_fmaf(entry_value(z, e) - base, a.l2e, -l2));
    if constexpr (sizeof(Tin) == 2) d[e] = to_bf16(o);
    else d[e] = o;
  }
}

// NT threads x NC chunks of a row in registers, KS x NT more in LDS. With PF the row after the next
// starts early: its first PF x NT chunks go straight to LDS while this row is worked on, the rest to
// registers once this row's stores are out. Vector memory operations are waited for in the order they
// were issued, so whatever a row waits for in its middle (the student's logits at the record's tokens,
// its single entries) is issued before those loads, from ids that were loaded a row earlier.
// The waves per SIMD are named since the compiler otherwise takes 149 registers where 127 do (NC = 16).
template <typename Tin, int NT, int NC, int KS, int PF, typename Sum>
__global__ __launch_bounds__(NT, NC == 4 ? 5 : NC == 24 ? 3 : 4) void distill_rows(DistillArgs a) {
  static_assert(PF <= NC && (KS == 0 || PF == 0));
  constexpr int KE = (kMaxK + NT - 1) / NT;   // entries of a record per thread: tid, tid + NT, ...
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int U = 4;                     // further chunks per thread in flight
  __shared__ float red[2][2 * (NT / 64)];
  constexpr int kRecs = NT == 64 ? 1 : 2;     // one wave is never in two rows
  __shared__ Record<NT> recs[kRecs];
  __shared__ RecordMath rm;
  __shared__ double far_red[NT / 64];
  __shared__ int far_rows;
  __shared__ u32x4 keep[KS > 0 ? KS * NT : 1];
  __shared__ u32x4 ahead[PF > 0 ? PF * NT : 1];   // [chunk][thread]: a wave reads what it loaded
  const int tid = threadIdx.x;
  const int V = a.V;
  const float L = a.l2e;
  recs[0].head[tid] = recs[kRecs - 1].head[tid] = -1;
  if (tid == 0) far_rows = 0;
  auto is_valid = [&](int64_t row) { return a.mask == nullptr || uload_u8(a.mask + row) != 0; };
  uint32_t r[NC][4];
  auto load_row = [&](int64_t row, bool rd) {
    const Tin* z = (const Tin*)a.logits + (rd ? row : 0) * a.ld;
    const RowSplit sp = split_row(z, V);
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead, rd ? sp.nfull * 16 : 0);
#pragma unroll
    for (int c = PF; c < NC; ++c) load16<kAuxLast>(r[c], rz, tid * 16, c * NT * 16);
  };
  auto load_ahead = [&](int64_t row, bool rd) {
    if constexpr (PF > 0) {
      const Tin* z = (const Tin*)a.logits + (rd ? row : 0) * a.ld;
      const RowSplit sp = split_row(z, V);
      const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead, rd ? sp.nfull * 16 : 0);
      const int wave0 = __builtin_amdgcn_readfirstlane(tid & ~63);
#pragma unroll
      for (int c = 0; c < PF; ++c)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rz, (__attribute__((address_space(3))) void*)&ahead[c * NT + wave0], 16, tid * 16, c * NT * 16, 0, kAuxLast);
    }
  };
  // one entry of a row (0 for e = -1), as bits of a float
  auto load_one = [&](__amdgpu_buffer_rsrc_t rz, int e) -> uint32_t {
    const int off = e < 0 ? 0x7fffff00 : e * (int)sizeof(Tin);
    if constexpr (sizeof(Tin) == 2) return __builtin_amdgcn_raw_buffer_load_b16(rz, off, 0, kAuxKeep);
    else return __builtin_amdgcn_raw_buffer_load_b32(rz, off, 0, kAuxKeep);
  };
  auto value_of = [&](uint32_t w) { return __uint_as_float(sizeof(Tin) == 2 ? w << 16 : w); };
  // this thread's entries of a row's record
  int id_next[KE];
  float tv_next[KE];
  auto load_entries = [&](int64_t row, bool rd) {
    const int64_t at = (rd ? row : 0) * a.k;
    const int bytes = rd ? a.k * 4 : 0;
    const __amdgpu_buffer_rsrc_t ri = row_rsrc(a.tokens + at, bytes), rv = row_rsrc(a.values + at, bytes);
#pragma unroll
    for (int i = 0; i < KE; ++i) {
      id_next[i] = (int)__builtin_amdgcn_raw_buffer_load_b32(ri, tid * 4, i * NT * 4, kAuxKeep);
      tv_next[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rv, tid * 4, i * NT * 4, kAuxKeep));
    }
  };
  auto unpack = [&](const auto& v, float (&x)[E]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(Tin) == 2) {
        x[2 * j] = bf16_lo(v[j]);
        x[2 * j + 1] = bf16_hi(v[j]);
      } else {
        x[j] = __uint_as_float(v[j]);
      }
    }
  };
  int64_t row = blockIdx.x;
  bool valid = row < a.T && is_valid(row);
  load_entries(row, valid);
  load_ahead(row, valid);
  load_row(row, valid);
  const float scale = call_scale<NT>(a);   // its loads in flight together with the first row's
  __syncthreads();                         // the lists are empty
  int parity = 0;                          // flips after each row that was evaluated
  for (; row < a.T; row += gridDim.x) {
    const int64_t next = row + gridDim.x;
    const bool next_valid = next < a.T && is_valid(next);
    Tin* drow = a.dlogits ? (Tin*)a.dlogits + row * a.ldd : nullptr;
    const Tin* zrow = (const Tin*)a.logits + row * a.ld;
    const RowSplit sp = split_row(zrow, V);
    const int nfull = sp.nfull;
    const bool edge = tid < sp.nedge;
    const int ei = sp.template entry<E>(tid);
    Record<NT>& rec = recs[kRecs == 1 ? 0 : parity];
    bool good = valid;
    // This thread's entries of the record (id, -1 for none; value; the student's logit) and its single
    // entry of the row.
    int id[KE];
    float tv[KE];
    uint32_t tz_word[KE];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < KE; ++i) {
      const bool in = valid && i * NT + tid < a.k;
      const bool out = in && (id_next[i] < -1 || id_next[i] >= V);
      bad |= out;
      id[i] = in && !out ? id_next[i] : -1;
      tv[i] = id[i] >= 0 ? tv_next[i] : -INFINITY;
    }
    if constexpr (PF > 0) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int c = 0; c < PF; ++c) {
        const u32x4 v = ahead[c * NT + tid];
        r[c][0] = v.x;
        r[c][1] = v.y;
        r[c][2] = v.z;
        r[c][3] = v.w;
      }
    }
    // without branches, and used only behind the first pass: a load that misses its row's range reads 0
    const __amdgpu_buffer_rsrc_t re = row_rsrc(zrow, V * (int)sizeof(Tin));
#pragma unroll
    for (int i = 0; i < KE; ++i) tz_word[i] = load_one(re, id[i]);
    const uint32_t xe_word = load_one(re, valid && edge ? ei : -1);
    load_entries(next, next_valid);
    if (valid) {
      // an entry goes to the list of the thread that owns its token
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        const int j = i * NT + tid;
        if (j >= a.k) break;
        rec.id[j] = id[i];
        rec.again[j] = 0;
        if (id[i] >= 0) {
          const int e = id[i] - sp.lead;
          const int owner = e >= 0 && e < nfull * E ? (e / E) % NT : (e < 0 ? id[i] : id[i] - nfull * E);
          rec.next[j] = (int16_t)atomicExch(&rec.head[owner], j);
        }
      }
      if (tid == 0) rm.any_again = 0;
      good = !__syncthreads_or(bad);       // a token outside the vocabulary makes the row bad
      parity ^= 1;
    }
    int head = -1;
    uint32_t slots = 0;                    // bit s mod 32: a record's token lies in chunk slot s
    bool edge_held = false;
    float xe = -INFINITY;                  // this thread's single entry
    // the record's entries of this thread's chunk of a slot: f(j, entry of the chunk). What depends
    // on the slot is uniform here and below: a value per slot and thread would be kept in a
    // register across the rows.
    auto held = [&](int slot, auto&& f) {
      for (int j = head; j >= 0; j = rec.next[j]) {
        const int e = rec.id[j] - (sp.lead + slot * NT * E) - tid * E;
        if (e >= 0 && e < E) f(j, e);
      }
    };
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(zrow + sp.lead, nfull * 16);
    if (!good) {                           // uniform
      if (valid) rec.head[tid] = -1;
      if (tid == 0) {
        a.loss_tok[row] = 0.0f;
        a.flags[row] = valid ? (uint8_t)(DPPO_FLAG_VALID | DPPO_FLAG_BAD_ID) : (uint8_t)0;
      }
    } else {
      head = rec.head[tid];
      rec.head[tid] = -1;                  // the list stays reachable through `head`
      for (int j = head; j >= 0; j = rec.next[j]) {
        const int e = rec.id[j] - sp.lead;
        if (e >= 0 && e < nfull * E) slots |= 1u << ((e / E / NT) & 31);
        else edge_held = true;
        for (int j2 = rec.next[j]; j2 >= 0; j2 = rec.next[j2])
          if (rec.id[j2] == rec.id[j]) {
            rec.again[j > j2 ? j : j2] = 1;
            rm.any_again = 1;
          }
      }
      float N = kNoShift;
      Sum sum = 0;
      auto add = [&](float (&x)[E], int slot) {
        if (slots >> (slot & 31) & 1u)
          held(slot, [&](int, int e) {
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = i == e ? -INFINITY : x[i];
          });
        float cm = max3(x[0], x[1], x[2]);
        if constexpr (E == 8) cm = max3(cm, max3(x[3], x[4], x[5]), max3(x[6], x[7], x[7]));
        else cm = fmaxf(cm, x[3]);
        add_logits(N, sum, x, cm, L);
      };
      // the chunks past the registers
      if constexpr (KS > 0) {
        for (int s0 = NC; s0 * NT < nfull; s0 += U) {
          u32x4 v[U];
#pragma unroll
          for (int u = 0; u < U; ++u) v[u] = buf_load16(rz, tid * 16, (s0 + u) * NT * 16);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (s0 + u - NC < KS) keep[(s0 + u - NC) * NT + tid] = v[u];
            if (tid >= nfull - (s0 + u) * NT) continue;
            float x[E];
            unpack(v[u], x);
            add(x, s0 + u);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (c * NT < nfull) {              // uniform
          float x[E];
          unpack(r[c], x);
          if (tid < nfull - c * NT) add(x, c);
        }
        // the words, not what was made of them, stay live until the gradient
        asm volatile("" : "+v"(r[c][0]), "+v"(r[c][1]), "+v"(r[c][2]), "+v"(r[c][3]));
        __builtin_amdgcn_sched_barrier(0);
      }
      xe = value_of(xe_word);
      if (edge) {
        bool own = false;
        if (edge_held)
          for (int j = head; j >= 0; j = rec.next[j]) own |= rec.id[j] == ei;
        const float x[1] = {own ? -INFINITY : xe};
        add_logits(N, sum, x, x[0], L);
      }
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        const int j = i * NT + tid;
        if (j >= a.k) break;
        rm.value[j] = tv[i];
        rm.z[j] = id[i] >= 0 ? value_of(tz_word[i]) : -INFINITY;
      }
      N = shift_of(N);
      float S = (float)sum;
      block_merge_ns_int<NT>(N, S, red[parity]);
      if (tid < 64) record_math(a, row, scale * (a.tscale ? uload(a.tscale + row) : 1.0f), N, S, rec, rm);
      if (tid == 0) {
        a.flags[row] = rm.far ? kFlagFar : (uint8_t)DPPO_FLAG_VALID;
        far_rows |= rm.far;
      }
      __syncthreads();
    }
    load_ahead(next, next_valid);
    if (!good) {
      if (drow) zero_row<Tin, NT>(drow, V);
    } else if (drow && !rm.far) {          // uniform
      {
        const float w = rm.w, l2 = rm.lse2;
        const __amdgpu_buffer_rsrc_t rd = row_rsrc(drow + sp.lead, nfull * 16);
        const bool same = (((uintptr_t)drow - (uintptr_t)zrow) & 15) == 0;    // uniform
        auto put = [&](const float (&x)[E], int slot) {
          float o[E];
#pragma unroll
          for (int i = 0; i < E; ++i) o[i] = w * exp2_hw(__builtin_fmaf(x[i], L, -l2));
          if (slots >> (slot & 31) & 1u)
            held(slot, [&](int j, int e) {
              if (rec.again[j]) return;
              const float gj = rec.grad[j];
#pragma unroll
              for (int i = 0; i < E; ++i) o[i] = i == e ? gj : o[i];
            });
          u32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(Tin) == 2) v[i] = pack_bf16(o[2 * i], o[2 * i + 1]);
            else v[i] = __float_as_uint(o[i]);
          }
          if (same) {
            buf_store16_nt(v, rd, tid * 16, slot * NT * 16);   // dropped past the row
          } else if (tid < nfull - slot * NT) {
            // dlogits at another offset within 16 bytes: entry by entry
            Tin* d = drow + (sp.lead + slot * NT * E) + tid * E;
#pragma unroll
            for (int i = 0; i < E; ++i) {
              if constexpr (sizeof(Tin) == 2) d[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
              else d[i] = __uint_as_float(v[i]);
            }
          }
        };
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (c * NT < nfull) {
            float x[E];
            unpack(r[c], x);
            put(x, c);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (KS > 0) {
          for (int s0 = NC; s0 * NT < nfull; s0 += U) {
            u32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if (s0 + u - NC < KS) v[u] = keep[(s0 + u - NC) * NT + tid];
              else v[u] = buf_load16<kAuxLast>(rz, tid * 16, (s0 + u) * NT * 16);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if ((s0 + u) * NT >= nfull) continue;
              float x[E];
              unpack(v[u], x);
              put(x, s0 + u);
            }
          }
        }
        if (edge) {
          float o = w * exp2_hw(__builtin_fmaf(xe, L, -l2));
          if (edge_held)
            for (int j = head; j >= 0; j = rec.next[j])
              if (rec.id[j] == ei && !rec.again[j]) o = rec.grad[j];
          if constexpr (sizeof(Tin) == 2) drow[ei] = to_bf16(o);
          else drow[ei] = o;
        }
      }
    }
    load_row(next, next_valid);
    valid = next_valid;
  }
  __syncthreads();
  if (far_rows) {                          // uniform
    for (row = blockIdx.x; row < a.T; row += gridDim.x)
      if (a.flags[row] == kFlagFar) far_row<Tin, NT>(a, row, scale, recs[0], rm, far_red);
  }
}

// The loss sum and the counters, in one workgroup. L is summed in float64, each thread over a fixed
// stride, then a fixed tree: the same inputs give the same bits on every run. (loss_sum, which also
// counts what the PPO decisions need, takes 7.5 us where this takes 4.)
__global__ __launch_bounds__(1024) void distill_sum(const float* kl, const uint8_t* flags, const float* tscale,
                                                    int32_t* stats, int64_t T, float loss_scale, int32_t scale_mode,
                                                    float* loss) {
  constexpr int U = 8;
  __shared__ double part[16];
  __shared__ int counts[2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double acc = 0.0;
  int n_valid = 0, n_bad = 0;              // this wave's
  for (int64_t base = threadIdx.x; base - lane < T; base += 1024 * U) {
    float l[U], ts[U];
    uint32_t f[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = base + (int64_t)u * 1024;
      const int64_t j = i < T ? i : T - 1;
      l[u] = kl[j];
      ts[u] = tscale ? tscale[j] : 1.0f;
      f[u] = i < T ? flags[j] : 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // masked and bad rows have l = 0, and must not meet a scale that is not finite
      if ((f[u] & (DPPO_FLAG_VALID | DPPO_FLAG_BAD_ID)) == DPPO_FLAG_VALID) acc += (double)ts[u] * (double)l[u];
      n_valid += __popcll(__ballot(f[u] & DPPO_FLAG_VALID));
      n_bad += __popcll(__ballot(f[u] & DPPO_FLAG_BAD_ID));
    }
  }
  acc = wave_sum_f64(acc);
  if (lane == 0) {
    part[wave] = acc;
    counts[0][wave] = n_valid;
    counts[1][wave] = n_bad;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    acc = wave_sum_f64(lane < 16 ? part[lane] : 0.0);
    int n = lane < 16 ? counts[0][lane] : 0, bad = lane < 16 ? counts[1][lane] : 0;
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) {
      n += __shfl_xor(n, off, 64);
      bad += __shfl_xor(bad, off, 64);
    }
    if (lane == 0) {
      const float scale = scale_mode == DPPO_SCALE_TOKEN_MEAN ? loss_scale / (float)(n > 1 ? n : 1) : loss_scale;
      loss[0] = (float)((double)scale * acc);
      for (int k = 0; k < DPPO_N_STATS; ++k) stats[k] = 0;
      stats[DPPO_STAT_N_VALID] = n;
      stats[DPPO_STAT_N_BAD] = bad;
    }
  }
}

constexpr int64_t kMaxGrid = 1 << 20;      // HIP holds a grid's threads to 32 bits

struct Shape {
  int nt;
  int64_t chunks;      // of the longest row it takes
  int rounds;          // workgroups per place on the device, 0: one per row
  const void *bf16, *f32;
};
// The loads ahead hide the record's arithmetic behind memory: with and without, us: bf16 k = 32, T = 4096,
// V = 106495 412 and 426, V = 155647 602 and 614; fp32 k = 128, T = 4096, V = 50257 401 and 415, though
// 377 and 371 at k = 32.
template <int NT, int NC, int KS, int PF, typename Sum = float>
constexpr Shape shape(int rounds, int64_t chunks = (int64_t)NT * NC) {
  return {NT, chunks, rounds, (const void*)distill_rows<uint16_t, NT, NC, KS, PF, Sum>,
          (const void*)distill_rows<float, NT, NC, KS, PF, Sum>};
}

}  // namespace

namespace {
// Workgroups of a kernel that fit on the current device at once; the query takes microseconds, so it
// is made once per device and kernel (more of them than the table holds are asked for each time).
hipError_t resident_groups(const void* fn, int threads, int64_t* groups) {
  struct Known {
    int dev;
    const void* fn;
    int64_t groups;
  };
  static std::mutex mu;
  static Known known[256];
  static int count = 0;
  int dev = 0, cus = 0, per_cu = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < count; ++i)
    if (known[i].dev == dev && known[i].fn == fn) {
      *groups = known[i].groups;
      return hipSuccess;
    }
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess) e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, threads, 0);
  if (e != hipSuccess) return e;
  *groups = (int64_t)cus * std::max(per_cu, 1);
  if (count < 256) known[count++] = {dev, fn, *groups};
  return hipSuccess;
}
}  // namespace

hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t st) {
  // The smallest shape that holds the row; the last two stream the rest of longer ones, with a thread's sum in
  // 32 bits up to 64 chunks (64 * 2^-24 = 3.8e-6) and in 64 bits for any length (2^15 equal chunks, at V =
  // 2^28, would be off by 5e-4; V = 300000 takes 529 us in 32 bits and 533 in 64). In bf16, T = 8192, by
  // the shape that is taken and by the next one, us: V = 4095 59 and 64, 8191 87 and 102, 32767 236 and
  // 263, 65535 452 and 556; V = 155647 at T = 4096 602 and 602.
  //
  // How many workgroups: one that takes row after row has the next row's loads in flight while it
  // stores, and pays its start once; workgroups that start as others end keep the compute units evenly
  // loaded. One workgroup per place / three per place / one per row, us: V = 4000 60 / 66 / 67 and 12000
  // 122 / 123 / 140, V = 28000 208 / 198 / 204 and 40000 277 / 274 / 284, V = 50257 378 / 366 / 367 and
  // 65535 476 / 461 / 452 (bf16, T = 8192), V = 106495 at T = 4096 412 / - / 451.
  static const Shape shapes[] = {
      shape<64, 4, 0, 0>(1),    shape<128, 4, 0, 0>(1),  shape<128, 8, 0, 0>(1),  shape<256, 8, 0, 0>(1),
      shape<256, 16, 0, 0>(3),  shape<256, 24, 0, 0>(3), shape<512, 16, 0, 0>(0), shape<1024, 13, 0, 8>(1),
      shape<1024, 19, 0, 8>(1), shape<1024, 16, 7, 0>(1, 64 * 1024),
      shape<1024, 16, 7, 0, double>(1, INT64_MAX)};
  const int64_t chunks = (int64_t)a.V * (bf16 ? 2 : 4) / 16;
  // Few rows leave most of the device idle and wait for one row's steps: more threads share its chunks.
  // 512 threads against the smallest shape, us, bf16: V = 32000 20 and 25 at T = 64, 27 and 30 at T = 512,
  // 46 and 40 at T = 1024; V = 10000 18 and 20 at T = 256, 34 and 25 at T = 1000.
  const int least = a.T <= 512 ? 512 : 64;
  const Shape* s = shapes;
  while (s + 1 < shapes + sizeof(shapes) / sizeof(shapes[0]) &&
         (s->chunks < chunks || s->nt < least))
    ++s;
  const void* fn = bf16 ? s->bf16 : s->f32;
  int64_t slots = 0;
  hipError_t e = resident_groups(fn, s->nt, &slots);
  if (e != hipSuccess) return e;
  const int64_t grid = std::min<int64_t>(a.T, s->rounds ? s->rounds * slots : kMaxGrid);
  DistillArgs args = a;
  void* kargs[] = {&args};
  e = hipLaunchKernel(fn, dim3((unsigned)grid), dim3((unsigned)s->nt), kargs, 0, st);
  return e == hipSuccess ? hipGetLastError() : e;
}

hipError_t launch_distill_sum(const DistillArgs& a, float* loss, hipStream_t st) {
  distill_sum<<<1, 1024, 0, st>>>(a.loss_tok, a.flags, a.tscale, a.stats, a.T, a.loss_scale, a.scale_mode, loss);
  return hipGetLastError();
}

}  // namespace dppo
