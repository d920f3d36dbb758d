// Token embedding with scaling and its gradient, gfx950.
//
//   y_t = scale W[id_t];  dW[v] = scale sum over t with id_t = v of dy_t
// An id outside 0 .. V - 1 is padding: a row of zeros, no gradient.  HBM-bound.

#include "packed.hpp"

#include "common.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256;

// tpr threads per token row (a power of two), kThreads / tpr rows per workgroup
__global__ void __launch_bounds__(kThreads)
embed_fwd_kernel(const int64_t* __restrict__ ids, const lt_half* __restrict__ W, int64_t ldw, float scale,
                 lt_half* __restrict__ Y, int64_t ldy, int64_t T, int nch, int64_t V, int tpr) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / tpr) + threadIdx.x / tpr;
  if (t >= T) return;
  const int64_t id = ids[t];
  const bool ok = id >= 0 && id < V;
  const lt_half* w = W + (ok ? id : 0) * ldw;
  for (int c = threadIdx.x % tpr; c < nch; c += tpr) {
    half8 v = as_half8(ok ? ld16(w + (int64_t)c * 8) : u32x4{0, 0, 0, 0});
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (_Float16)((float)v[e] * scale);
    st16(Y + t * ldy + (int64_t)c * 8, as_u32x4(v));
  }
}

// One workgroup per (row of the table, 2048 columns): it goes through the ids
// 256 at a time and adds the rows of its tokens in order.
__global__ void __launch_bounds__(kThreads)
embed_bwd_kernel(const EmbedBwdArgs a) {
  __shared__ int hits[kThreads];
  __shared__ int counts[kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t v = blockIdx.x;
  const int64_t c0 = ((int64_t)blockIdx.y * kThreads + tid) * 8;
  const bool in = c0 < a.H;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bool any = false;
  for (int64_t t0 = 0; t0 < a.T; t0 += kThreads) {
    const bool hit = t0 + tid < a.T && a.ids[t0 + tid] == v;
    const uint64_t bal = __builtin_amdgcn_ballot_w64(hit);
    if (lane == 0) counts[wave] = __popcll(bal);
    __syncthreads();
    int at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) at += counts[w];
      n += counts[w];
    }
    if (hit) hits[at + __popcll(bal & ((1ull << lane) - 1))] = tid;
    __syncthreads();
    any |= n > 0;
    for (int k = 0; k < n; ++k) {
      if (in) {
        const half8 g = as_half8(ld16(a.dY + (t0 + hits[k]) * a.lddy + c0));
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += (float)g[e];
      }
    }
    __syncthreads();
  }
  if (!in || (a.accumulate && !any)) return;
  lt_half* dst = a.dW + v * a.lddw + c0;
  half8 o;
  if (a.accumulate) {
    o = as_half8(ld16(dst));
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (_Float16)((float)o[e] + acc[e] * a.scale);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (_Float16)(acc[e] * a.scale);
  }
  st16(dst, as_u32x4(o));
}

}  // namespace

hipError_t embed_fwd_launch(const int64_t* ids, const lt_half* W, int64_t ldw, float scale, lt_half* Y, int64_t ldy,
                            int64_t T, int64_t H, int64_t V, hipStream_t s) {
  const int nch = (int)(H / 8);
  int tpr = 8;
  while (tpr < nch && tpr < kThreads) tpr *= 2;
  const int64_t rpb = kThreads / tpr;
  hipLaunchKernelGGL(embed_fwd_kernel, dim3((unsigned)((T + rpb - 1) / rpb)), dim3(kThreads), 0, s, ids, W, ldw,
                     scale, Y, ldy, T, nch, V, tpr);
  return hipGetLastError();
}

hipError_t embed_bwd_launch(const EmbedBwdArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.V, (unsigned)((a.H + kThreads * 8 - 1) / (kThreads * 8)));
  hipLaunchKernelGGL(embed_bwd_kernel, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace lt
