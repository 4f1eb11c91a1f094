// The k largest logits of every row, best first (equal values by index), with the row's
// log-sum-exp: one read of the logits.
//
// A bound that at least k entries reach lets almost every entry be dropped with one comparison. The
// k-th largest of the threads' running maxima is such a bound: k different entries reach it. A
// workgroup streams a row in tiles of U 16-byte chunks per thread; after the first tile, and each
// time the part read has doubled, it takes that bound from the maxima so far, and chunks with an entry
// that reaches the bound of their time are kept in LDS (about k (1 + ln tiles) of them in random
// order). At the end the kept chunks' entries that reach the last bound are ranked by counting. What the
// fast path cannot hold (long runs of equal values, a row with NaN or infinities, fewer than k finite
// entries) is selected exactly by radix passes over the row.
//
// Long rows in a batch that fills the device are bound by HBM: T = 8192, V = 151936 bf16, k = 64 takes 437
// us, 5.7 TB/s of logits; T = 2048, V = 50257 fp32, k = 128 takes 91 us, 4.5 TB/s, a quarter of it the
// starts and ends of rows of 25 chunks a thread. One row (V = 262144 fp32, 16 parts and a join, 20 us) and
// decode batches (T = 8, V = 32000 bf16, 12 us) are chains of a few loads, barriers and the ranking.
#include "top_logits.h"

#include <algorithm>

#include "dppo.h"
#include "dppo_device.h"
#include "f64_math.h"
#include "row_split.h"

namespace dppo {

namespace {

// 16-byte chunks per thread in flight. Four leave 64 registers and LDS for 32 waves per CU: against
// eight (24 waves) T = 8192, V = 151936 bf16, k = 64 497 -> 436 us, T = 2048, V = 50257 fp32, k = 128
// 120 -> 94 us.
constexpr int kTopU = 4;
// Kept chunks, and entries of them that reach the final bound. A row whose maxima are too few for a
// bound is kept whole: fewer than 256 chunks of 8 entries and two ends.
constexpr int kTopChunks = 1056;
constexpr int kTopCap = 2112;
constexpr int kTopRank = 512;    // more than these are thinned out before the ranking

// Unsigned keys in the order of the values: -0 as +0, NaN above +inf.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  if (x != x) return 0xFFFFFFFFu;
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xFFFFFFFFu) return __builtin_nanf("");
  return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k);
}
constexpr uint32_t kKeyLowest = 0x00800000u;  // the key of -FLT_MAX

// Larger value first, then the lower index.
__device__ __forceinline__ uint64_t composite(float x, int idx) {
  return ((uint64_t)value_key(x) << 32) | (uint32_t)~idx;
}

template <typename Tin>
__device__ __forceinline__ float entry_value(const Tin* p, int64_t i) {
  if constexpr (sizeof(Tin) == 2) return bf16_to_f32(p[i]);
  else return p[i];
}

template <typename Tin>
__device__ __forceinline__ void unpack(const uint32_t (&r)[4], float (&x)[16 / sizeof(Tin)]) {
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
  else return max3(max3(x[0], x[1], x[2]), x[3], x[3]);
}

// Output slot `rank` of a row (or of a row's part).
__device__ __forceinline__ void put(const TopArgs& a, int64_t row, int part, int rank, uint64_t c) {
  if (a.parts > 1) {
    a.cand[(row * a.parts + part) * a.k + rank] = c;
  } else {
    a.values[row * a.k + rank] = key_value((uint32_t)(c >> 32));
    a.ids[row * a.k + rank] = (int32_t)~(uint32_t)c;
  }
}

// Sorts list[0, n), n <= 64 R, best first, by one wave: a bitonic network over R entries per lane in
// registers (place lane R + r). Ranking by counting took n / 64 passes over the list instead: at k =
// 250 most of a short row's time.
template <int R>
__device__ __noinline__ void sort_list(uint64_t* list, int n) {
  const int lane = threadIdx.x & 63;
  uint64_t v[R];
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = lane * R + r < n ? list[lane * R + r] : 0;
#pragma unroll
  for (int size = 2; size <= 64 * R; size *= 2) {
#pragma unroll
    for (int stride = size / 2; stride > 0; stride /= 2) {
      if (stride >= R) {
        const int mask = stride / R;
        const bool lower = (lane & mask) == 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const bool down = ((lane * R + r) & size) == 0;      // this run of `size` falls
          const uint64_t o = __shfl_xor(v[r], mask, 64);
          v[r] = (v[r] > o) == (lower == down) ? v[r] : o;
        }
      } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r & stride) continue;
          const bool down = ((lane * R + r) & size) == 0;
          const uint64_t x = v[r], y = v[r + stride];
          const bool swap = (x > y) != down;
          v[r] = swap ? y : x;
          v[r + stride] = swap ? x : y;
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (lane * R + r < n) list[lane * R + r] = v[r];
}
constexpr int kSortMost = 512;
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  if (n <= 64) sort_list<1>(list, n);
  else if (n <= 128) sort_list<2>(list, n);
  else if (n <= 256) sort_list<4>(list, n);
  else sort_list<8>(list, n);
}

// Exactly the kk best of the entries [e0, e1) of z into cand, in any order: the key of the kk-th by radix
// passes over the row, then everything above it and the first of its equals. By the whole workgroup,
// behind a barrier; hist holds 256 counts, wcount one per wave. (Sum is the calling kernel's: a copy for
// each, since one that two kernels share costs the fp32 rows two spilled registers, 94 -> 99 us at T = 2048, V
// = 50257.)
template <typename Tin, int NT, typename Sum>
__device__ __noinline__ void select_exact(const Tin* z, int e0, int e1, int kk, uint64_t* cand, int* count,
                                          int* hist, int* wcount) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  uint32_t prefix = 0, mask = 0;
  int need = kk;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    for (int e = e0 + tid; e < e1; e += NT) {
      const uint32_t key = value_key(entry_value(z, e));
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255u], 1);
    }
    __syncthreads();
    int bin = 255;
    for (int above = hist[bin]; above < need; above = hist[bin]) {
      need -= above;
      --bin;
    }
    prefix |= (uint32_t)bin << shift;
    mask |= 255u << shift;
    __syncthreads();
  }
  if (tid == 0) *count = 0;
  int before = 0;                          // equals before this step
  __syncthreads();
  for (int base = e0; base < e1; base += NT) {
    const int e = base + tid;
    const float x = e < e1 ? entry_value(z, e) : 0.0f;
    const uint32_t key = value_key(x);
    const bool tie = e < e1 && key == prefix;
    const uint64_t ties = __ballot(tie);
    if (lane == 0) wcount[wave] = __popcll(ties);
    __syncthreads();
    int at = before + __popcll(ties & ((1ull << lane) - 1ull));
    for (int w = 0; w < NW; ++w) {
      if (w < wave) at += wcount[w];
      before += wcount[w];
    }
    if ((e < e1 && key > prefix) || (tie && at < need)) cand[atomicAdd(count, 1)] = composite(x, e);
    __syncthreads();
  }
}

// Whether a row's sum 2^N S in 32 bits is its sum of exponentials (uniform).
__device__ __forceinline__ bool near_row(float N, float S) { return S > 0.0f && S < INFINITY && fabsf(N) < kFarLog2; }

// The log-sum-exp of a far row, around its maximum in 64 bits; NaN for a row holding NaN or +inf, or only
// -inf. By the whole workgroup; red holds a double per wave, and is free on return.
template <typename Tin, int NT>
__device__ __noinline__ float far_lse(const Tin* z, int V, double t2e, double* red) {
  constexpr int NW = NT / 64;
  const int wave = threadIdx.x >> 6;
  float m = -INFINITY;
  for (int e = threadIdx.x; e < V; e += NT) {
    const float x = entry_value(z, e);
    m = x != x ? INFINITY : fmaxf(m, x);
  }
  m = wave_max(m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave] = m;
  __syncthreads();
  double M = red[0];
  for (int w = 1; w < NW; ++w) M = fmax(M, red[w]);
  __syncthreads();
  if (fabs(M) == INFINITY) return __builtin_nanf("");
  double s = 0.0;
  for (int e = threadIdx.x; e < V; e += NT) s += exp2_f64(((double)entry_value(z, e) - M) * t2e);
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) red[wave] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < NW; ++w) s += red[w];
  __syncthreads();
  return (float)(__builtin_fma(M, t2e, log2_f64(s)) * kLn2F64);
}

// Sum: what a thread's sum of exponentials is held in. 64 chunks a thread in 32 bits cost it 64 * 2^-24 =
// 3.8e-6; 8192 equal ones (V = 2^28 in 16 parts) would be off by 1e-4. T = 8192, V = 151936 bf16: 436 us in
// 32 bits, 443 in 64.
constexpr int kSumChunks = 64;
template <typename Tin, int NT, typename Sum>
__global__ __launch_bounds__(NT, 8) void top_rows(TopArgs a) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr int U = kTopU;
  constexpr int NW = NT / 64;
  __shared__ u32x4 chunk[kTopChunks];     // kept chunks; later the thinned-out entries
  __shared__ int chunk_at[kTopChunks];    // entry that a kept chunk starts at
  __shared__ uint64_t cand[kTopCap];
  __shared__ alignas(16) uint32_t tkey[NT];
  __shared__ float red[2 * NW];
  __shared__ int wcount[NW];
  __shared__ int chunks, chunks_s, count, kcount;
  __shared__ uint32_t bound_s;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int k = a.k;
  const float L = a.l2e;
  for (int64_t item = blockIdx.x; item < (int64_t)a.T * a.parts; item += gridDim.x) {
    const int64_t row = item / a.parts;
    const int part = (int)(item - row * a.parts);
    const Tin* z = (const Tin*)a.logits + row * a.ld;
    const RowSplit sp = split_row(z, a.V);
    // this part's chunks [c0, c0 + n), and the row's single entries at its ends
    const int c0 = (int)((int64_t)sp.nfull * part / a.parts);
    const int n = (int)((int64_t)sp.nfull * (part + 1) / a.parts) - c0;
    const int first = sp.lead + c0 * E;
    const int le = part == 0 ? sp.lead : 0;
    const int te = part == a.parts - 1 ? sp.nedge - sp.lead : 0;
    const int e0 = part == 0 ? 0 : first;                      // the part's entries [e0, e1)
    const int e1 = part == a.parts - 1 ? a.V : first + n * E;
    const bool edge = tid < le + te;
    const int ei = tid < le ? tid : sp.lead + sp.nfull * E + (tid - le);
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + first, n * 16);
    __syncthreads();                       // the last item's LDS is free
    if (tid == 0) chunks = count = kcount = 0;

    uint32_t r[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) load16<kAuxLast>(r[u], rz, tid * 16, u * NT * 16);
    float N = kNoShift, tmax = -INFINITY;
    Sum sum = 0;
    auto add = [&](const auto& x, float cm) {
      add_logits(N, sum, x, cm, L);
      tmax = fmaxf(tmax, cm);
    };
    float xe = -INFINITY;
    if (edge) {
      xe = entry_value(z, ei);
      const float x[1] = {xe};
      add(x, xe);
    }
    // the bound: the largest 16-bit key prefix that k threads' maxima reach
    auto update_bound = [&]() -> float {
      tkey[tid] = value_key(tmax);
      __syncthreads();
      if (wave == 0) {
        uint32_t key[NW];
#pragma unroll
        for (int j = 0; j < NW; ++j) key[j] = tkey[j * 64 + lane];
        uint32_t b = 0;
        for (int bit = 31; bit >= 16; --bit) {
          const uint32_t t = b | (1u << bit);
          int c = 0;
#pragma unroll
          for (int j = 0; j < NW; ++j) c += __popcll(__ballot(key[j] >= t));
          if (c >= k) b = t;
        }
        if (lane == 0) {
          bound_s = b > kKeyLowest ? b : kKeyLowest;
          chunks_s = chunks;               // between the barriers: nothing is kept meanwhile
        }
      }
      __syncthreads();
      return key_value(bound_s);
    };
    auto push = [&](float x, int idx) {
      const int slot = atomicAdd(&count, 1);
      if (slot < kTopCap) cand[slot] = composite(x, idx);
    };
    float bound = 0.0f;
    bool lost = false;                     // the list of chunks was full
    auto keep = [&](const uint32_t (&w)[4], float cm, int at) {
      if (cm >= bound) {
        const int slot = atomicAdd(&chunks, 1);
        if (slot < kTopChunks) {
          chunk[slot] = u32x4{w[0], w[1], w[2], w[3]};
          chunk_at[slot] = at;
        }
      }
    };
    auto test = [&](const uint32_t (&w)[4], float cm, int c) { keep(w, cm, first + c * E); };
    // first tile: the maxima, their bound, then the entries that reach it
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * NT >= n) break;              // uniform
      float x[E];
      unpack<Tin>(r[u], x);
      if (tid < n - u * NT) add(x, max_of(x));
    }
    bound = update_bound();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * NT >= n) break;
      float x[E];
      unpack<Tin>(r[u], x);
      if (tid < n - u * NT) test(r[u], max_of(x), u * NT + tid);
      if ((U + u) * NT < n) load16<kAuxLast>(r[u], rz, tid * 16, (U + u) * NT * 16);
    }
    int t = 1;
    for (int b = U * NT; b < n; b += U * NT, ++t) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (b + u * NT >= n) break;
        float x[E];
        unpack<Tin>(r[u], x);
        if (tid < n - b - u * NT) {
          const float cm = max_of(x);
          add(x, cm);
          test(r[u], cm, b + u * NT + tid);
        }
        if (b + (U + u) * NT < n) load16<kAuxLast>(r[u], rz, tid * 16, (b + (U + u) * NT) * 16);
      }
      if ((t & (t + 1)) == 0 && b + U * NT < n) {
        bound = update_bound();
        // drop kept chunks that no longer reach the bound before the list gets full
        const int have = chunks_s;
        if (have > kTopChunks / 2) {         // uniform
          lost |= have > kTopChunks;
          // in place: a step's chunks are read before any is kept, at places read already
          for (int i = 0; i < min(have, kTopChunks); i += NT) {
            const int j = i + tid;
            u32x4 v = {0u, 0u, 0u, 0u};
            int at = -1;
            if (j < min(have, kTopChunks)) {
              v = chunk[j];
              at = chunk_at[j];
            }
            __syncthreads();
            if (i == 0) {
              if (tid == 0) chunks = 0;
              __syncthreads();
            }
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            float x[E];
            unpack<Tin>(w, x);
            if (at >= 0) keep(w, max_of(x), at);
          }
        }
      }
    }
    if (n > U * NT) bound = update_bound();
    N = shift_of(N);
    float S = (float)sum;
    block_merge_ns_int<NT>(N, S, red);     // its barrier also makes the kept chunks final
    // the entries that reach the last bound
    const int nc = chunks;
    if (edge && xe >= bound) push(xe, ei);
    for (int i = tid; i < min(nc, kTopChunks); i += NT) {
      const u32x4 v = chunk[i];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      const int at = chunk_at[i];
      float x[E];
      unpack<Tin>(w, x);
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (x[j] >= bound) push(x[j], at + j);
    }
    __syncthreads();
    int m = count;
    uint64_t* list = cand;
    const int kk = k < e1 - e0 ? k : e1 - e0;
    if (lost || nc > kTopChunks || m > kTopCap || m < kk || !(S < INFINITY)) {
      __syncthreads();
      static_assert(NT >= 256);
      select_exact<Tin, NT, Sum>(z, e0, e1, kk, cand, &count, (int*)tkey, wcount);
      m = kk;
    } else if (m > kTopRank) {
      // thin out: a key that at least k and, if the keys allow it, at most kTopRank entries reach
      uint32_t b = 0;
      int reach = m;
      for (int bit = 31; bit >= 0 && reach > kTopRank; --bit) {
        const uint32_t key = b | (1u << bit);
        int c = 0;
        for (int i = tid; i < m; i += NT) c += (uint32_t)(cand[i] >> 32) >= key;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
        if (lane == 0) wcount[wave] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < NW; ++w) c += wcount[w];
        __syncthreads();
        if (c >= k) {
          b = key;
          reach = c;
        }
      }
      uint64_t* kept = (uint64_t*)chunk;
      static_assert(sizeof(chunk) >= 8 * kTopCap);
      for (int i = tid; i < m; i += NT) {
        const uint64_t c = cand[i];
        if ((uint32_t)(c >> 32) >= b) kept[atomicAdd(&kcount, 1)] = c;
      }
      __syncthreads();
      list = kept;
      m = kcount;
    }
    // By counting, which all waves share and which needs no registers: with the short rows' sort in this
    // kernel too its streaming loop has fewer (T = 8192, V = 151936, k = 64 440 -> 513 us; T = 4096,
    // k = 256 316 -> 288 us).
    for (int i = tid; i < m; i += NT) {
      const uint64_t c = list[i];
      int rank = 0;
      for (int j = 0; j < m; ++j) rank += list[j] > c;
      if (rank < k) put(a, row, part, rank, c);
    }
    for (int i = kk + tid; i < k; i += NT) put(a, row, part, i, 0);   // a part shorter than k
    if (a.parts > 1) {
      if (tid == 0) {
        a.part[2 * item] = N;
        a.part[2 * item + 1] = S;
      }
    } else {
      float lse = (N + log2f(S)) * kLn2;
      if (!near_row(N, S)) lse = far_lse<Tin, NT>(z, a.V, a.t2e, (double*)tkey);
      if (tid == 0) a.lse[row] = lse;
    }
  }
}

// ---------------------------------------------------------------------------------------
// Short rows: a wave per row, which stays in registers (M chunks per lane). No barriers, and up to 32
// rows of a CU in flight: T = 8192, V = 2048 bf16, k = 64 took 93 us with a workgroup per row. The
// bound is searched over the chunks' maxima (64 M groups), and where that leaves too many entries (few
// chunks, or k close to their number) over the entries themselves.
// ---------------------------------------------------------------------------------------
constexpr int kShortCap = 512;

template <typename Tin, int M>
__global__ __launch_bounds__(64) void top_short(TopArgs a) {
  constexpr int E = 16 / (int)sizeof(Tin);
  constexpr uint32_t kKeyInf = 0xFF800000u;          // the key of +inf
  __shared__ uint64_t cand[kShortCap];
  __shared__ alignas(16) int hist[256];
  __shared__ int count, wcount;
  const int lane = threadIdx.x;
  const uint64_t below = (1ull << lane) - 1ull;
  const int k = a.k;
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const Tin* z = (const Tin*)a.logits + row * a.ld;
    const RowSplit sp = split_row(z, a.V);
    const __amdgpu_buffer_rsrc_t rz = row_rsrc(z + sp.lead, sp.nfull * 16);
    uint32_t r[M][4];
#pragma unroll
    for (int m = 0; m < M; ++m) load16<kAuxLast>(r[m], rz, lane * 16, m * 1024);
    const bool edge = lane < sp.nedge;
    const int ei = sp.template entry<E>(lane);
    const float xe = edge ? entry_value(z, ei) : -INFINITY;
    float N = kNoShift, S = 0.0f;
    {
      const float x[1] = {xe};
      add_logits(N, S, x, xe, a.l2e);
    }
    float cm[M];                           // the chunks' maxima
#pragma unroll
    for (int m = 0; m < M; ++m) {
      cm[m] = -INFINITY;
      if (m * 64 >= sp.nfull) continue;    // uniform
      float x[E];
      unpack<Tin>(r[m], x);
      if (lane < sp.nfull - m * 64) {
        cm[m] = max_of(x);
        add_logits(N, S, x, cm[m], a.l2e);
      }
    }
    N = shift_of(N);
    wave_merge_ns_int(N, S);
    auto groups = [&](float f) {
      int c = __popcll(__ballot(xe >= f));
#pragma unroll
      for (int m = 0; m < M; ++m) c += __popcll(__ballot(cm[m] >= f));
      return c;
    };
    // entries that reach f: g(their lanes, value, entry), and how many
    auto entries = [&](float f, auto&& g) {
      uint64_t on = __ballot(xe >= f);
      int c = __popcll(on);
      g(on, 0, xe, ei);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if (__ballot(cm[m] >= f) == 0) continue;
        float x[E];
        unpack<Tin>(r[m], x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          on = __ballot(cm[m] >= f && x[j] >= f);    // a chunk outside the row has cm = -inf
          g(on, c, x[j], sp.lead + (m * 64 + lane) * E + j);
          c += __popcll(on);
        }
      }
      return c;
    };
    auto none = [](uint64_t, int, float, int) {};
    // largest key prefix found that enough groups, then entries, reach
    uint32_t lo = kKeyLowest, hi = kKeyInf;
    if (groups(key_value(lo)) >= k) {
      while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = groups(key_value(mid));
        if (c < k) {
          hi = mid;
        } else {
          lo = mid;
          if (c <= k + k / 8 + 2) break;
        }
      }
    }
    int n = entries(key_value(lo), none);
    const int most = k + k / 4 + 32;       // at most kShortCap
    static_assert(DPPO_MAX_TOP + DPPO_MAX_TOP / 4 + 32 <= kShortCap);
    if (S < INFINITY) {                    // uniform, like all of this
      hi = kKeyInf;
      while (n > most && hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = entries(key_value(mid), none);
        if (c < k) {
          hi = mid;
        } else {
          lo = mid;
          n = c;
        }
      }
    }
    if (!(S < INFINITY) || n > kShortCap || n < k) {
      __syncthreads();
      select_exact<Tin, 64, float>(z, 0, a.V, k, cand, &count, hist, &wcount);
      n = k;
    } else {
      entries(key_value(lo), [&](uint64_t on, int before, float x, int e) {
        if (on >> lane & 1ull) cand[before + __popcll(on & below)] = composite(x, e);
      });
    }
    __syncthreads();
    sort_list(cand, n);
    __syncthreads();
    for (int i = lane; i < k; i += 64) put(a, row, 0, i, cand[i]);
    float lse = (N + log2f(S)) * kLn2;
    if (!near_row(N, S)) lse = far_lse<Tin, 64>(z, a.V, a.t2e, (double*)hist);
    if (lane == 0) a.lse[row] = lse;
    __syncthreads();                       // cand is read
  }
}

// Joins a row's parts. Their lists are sorted, so the least of the parts' ceil(k / parts)-th entries is
// a bound that at least k entries reach; those are sorted.
constexpr int kJoinNT = 512;
constexpr int kTopParts = 16;

template <typename Tin>
__global__ __launch_bounds__(kJoinNT) void top_join(TopArgs a) {
  __shared__ uint64_t list[kTopParts * DPPO_MAX_TOP];
  __shared__ uint64_t kept[kTopParts * DPPO_MAX_TOP];
  __shared__ double red[kJoinNT / 64];
  __shared__ int count;
  const int tid = threadIdx.x;
  const int k = a.k;
  const int m = a.parts * k;
  const int share = (k + a.parts - 1) / a.parts;
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    __syncthreads();
    if (tid == 0) count = 0;
    for (int i = tid; i < m; i += kJoinNT) list[i] = a.cand[row * m + i];
    float N = -INFINITY, S = 0.0f;         // the same in every thread
    for (int p = 0; p < a.parts; ++p)
      merge_ns_int(N, S, a.part[2 * (row * a.parts + p)], a.part[2 * (row * a.parts + p) + 1]);
    __syncthreads();
    uint64_t bound = list[share - 1];
    for (int p = 1; p < a.parts; ++p) {
      const uint64_t c = list[p * k + share - 1];
      bound = c < bound ? c : bound;
    }
    for (int i = tid; i < m; i += kJoinNT) {
      const uint64_t c = list[i];
      if (c >= bound && c != 0) kept[atomicAdd(&count, 1)] = c;
    }
    __syncthreads();
    const int n = count;
    auto put = [&](int rank, uint64_t c) {
      a.values[row * k + rank] = key_value((uint32_t)(c >> 32));
      a.ids[row * k + rank] = (int32_t)~(uint32_t)c;
    };
    if (n <= kSortMost) {
      if (tid < 64) sort_list(kept, n);
      __syncthreads();
      for (int i = tid; i < k; i += kJoinNT) put(i, kept[i]);
    } else {
      for (int i = tid; i < n; i += kJoinNT) {
        const uint64_t c = kept[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += kept[j] > c;
        if (rank < k) put(rank, c);
      }
    }
    float lse = (N + log2f(S)) * kLn2;
    if (!near_row(N, S)) lse = far_lse<Tin, kJoinNT>((const Tin*)a.logits + row * a.ld, a.V, a.t2e, red);
    if (tid == 0) a.lse[row] = lse;
  }
}

}  // namespace

int top_parts(int64_t T, int64_t V, int es, int k) {
  // Parts of at least 2048 chunks and 16 chunks per entry asked for (a part brings k candidates to the
  // join), while the rows do not fill the device four times. us, bf16: at least 2048 and 4096 chunks 21
  // and 24 at T = 8, V = 151936, k = 64, 38 and 32 at T = 1, V = 33000, k = 256; 1024, 512 and 2048
  // workgroups 40, 49 and 51 at T = 200, V = 262144, 65, 67 and 88 at T = 1000, V = 151936.
  const int64_t least = std::max(2048, 16 * k);
  const int64_t most = std::min<int64_t>(kTopParts, V * es / (16 * least));
  const int64_t want = T > 0 ? 1024 / T : 1;
  return (int)std::max<int64_t>(1, std::min(most, want));
}

hipError_t launch_top_logits(const TopArgs& a, bool bf16, hipStream_t st) {
  constexpr int NT = 512;
  const int64_t items = (int64_t)a.T * a.parts;
  const int64_t chunks = (int64_t)a.V * (bf16 ? 2 : 4) / 16;
  // A wave per row where there are many short ones. Against a workgroup per row, us, bf16: 256 chunks
  // (V = 2000, k = 200) 21 and 28 at T = 300, 24 and 68 at T = 2000; 1000 chunks (V = 8000) with k = 20 28
  // and 24 at T = 2000, 68 and 76 at T = 8192, with k = 200 37 and 52, 97 and 180.
  if (chunks <= 64 * 16 && a.T >= (chunks <= 64 * 4 ? 256 : 2048)) {   // top_parts gives 1
    const unsigned g = (unsigned)std::min<int64_t>(a.T, kLaunchThreads / 64);
    if (chunks <= 64 * 4) {
      if (bf16) top_short<uint16_t, 4><<<g, 64, 0, st>>>(a);
      else top_short<float, 4><<<g, 64, 0, st>>>(a);
    } else {
      if (bf16) top_short<uint16_t, 16><<<g, 64, 0, st>>>(a);
      else top_short<float, 16><<<g, 64, 0, st>>>(a);
    }
    return hipGetLastError();
  }
  const int64_t grid = std::min<int64_t>(items, kLaunchThreads / NT);
  const dim3 g((unsigned)grid);
  if (chunks <= (int64_t)kSumChunks * NT * a.parts) {
    if (bf16) top_rows<uint16_t, NT, float><<<g, NT, 0, st>>>(a);
    else top_rows<float, NT, float><<<g, NT, 0, st>>>(a);
  } else {
    if (bf16) top_rows<uint16_t, NT, double><<<g, NT, 0, st>>>(a);
    else top_rows<float, NT, double><<<g, NT, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.parts > 1) {
    const int64_t g = std::min<int64_t>(a.T, kLaunchThreads / kJoinNT);
    if (bf16) top_join<uint16_t><<<dim3((unsigned)g), kJoinNT, 0, st>>>(a);
    else top_join<float><<<dim3((unsigned)g), kJoinNT, 0, st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace dppo
