// What the row kernels of the loss calls share: the call's scale and the zeros of a row that is not
// evaluated.
#pragma once

#include "dppo_device.h"
#include "loss_stage.h"
#include "row_split.h"
#include "token_math.h"

namespace dppo {

// The call's loss scale (Eq. 2: the token-mean normaliser, or the constant), once per
// workgroup; every thread calls it. Normally prep_stats has stored the valid-token count; in
// count mode the workgroup counts the mask itself (workgroup 0 also stores the count, for
// loss_sum), which saves that launch for a short batch. The short-row kernels and the fp32
// resident kernel (before their first row) and the bf16 kernels with two row buffers (behind
// their first row's loads) take this path; in the single-buffer bf16 kernels the extra prologue
// cost 0.7 % of the flagship's time even with count mode off. Counting behind the first row's
// loads in the fp32 kernel too was measured slower (the tiny batch's step 27.5 us against 25.6).
template <int NT>
__device__ float call_scale(const RowArgs& a) {
  if (a.mode == kModeLogprob) return 1.0f;
  if (!a.count_mode) return row_scale(a);
  if (a.scale_mode != DPPO_SCALE_TOKEN_MEAN) return a.loss_scale;
  __shared__ int part[NT / 64];
  int cnt = 0;
  if (a.mask != nullptr) {
    // 16-byte chunks from the 16-byte boundary at or below the mask, four per thread in
    // flight (T <= kCountModeMaxT); a byte counts when it lies in [mask, mask + T)
    const uintptr_t m0 = (uintptr_t)a.mask;
    const int ph = (int)(m0 & 15u);
    const int nb = ph + a.T;
    // The range check drops a 4-byte word that reaches past the resource's end, so the
    // resource runs to the next 4-byte boundary (readable, see the mask's requirement in the
    // ABI); bytes past the mask are not counted.
    const __amdgpu_buffer_rsrc_t r =
        row_rsrc((const void*)(m0 - (uintptr_t)ph), (nb + 3) & ~3);
    const int nch = (nb + 15) >> 4;
    for (int c0 = threadIdx.x; c0 < nch; c0 += 4 * NT) {
      u32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = c0 + u * NT;
        v[u] = buf_load16(r, c < nch ? c * 16 : 0x7fffff00, 0);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int base = (c0 + u * NT) * 16;
#pragma unroll
        for (int b = 0; b < 16; ++b) {
          const int pos = base + b;
          const uint32_t byte = (v[u][b >> 2] >> (8 * (b & 3))) & 0xffu;
          cnt += (byte != 0u) & (pos >= ph) & (pos < nb);
        }
      }
    }
  } else if (threadIdx.x == 0) {
    cnt = a.T;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) cnt += __shfl_xor(cnt, off, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = cnt;
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) n += part[i];
  if (blockIdx.x == 0 && threadIdx.x == 0) a.stats[DPPO_STAT_N_VALID] = n;
  return a.loss_scale / (float)(n > 1 ? n : 1);
}

// Zeros for a gradient row of V entries at any alignment: 16-byte stores over the whole chunks
// inside it, single entries before and after them.
template <typename Tin, int NT>
__device__ void zero_row(Tin* d, int V) {
  constexpr int E = 16 / (int)sizeof(Tin);
  const RowSplit sp = split_row(d, V);
  const u32x4 z = {0u, 0u, 0u, 0u};
  for (int i = threadIdx.x; i < sp.nfull; i += NT) __builtin_nontemporal_store(z, (u32x4*)(d + sp.lead) + i);
  if ((int)threadIdx.x < sp.nedge) d[sp.entry<E>(threadIdx.x)] = (Tin)0;
}

}  // namespace dppo
