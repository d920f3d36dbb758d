// Token embedding with scaling and its gradient, gfx950.
//
//   y_t = scale W[id_t];  dW[v] = scale sum over t with id_t = v of dy_t
// An id outside 0 .. V - 1 is padding: a row of zeros, no gradient.  HBM-bound: the
// rows that the tokens name in and Y out; dY in once and dW (all V rows, or with
// accumulation those of the tokens) out once.
//
// The gradient sorts the tokens by row, so that every row of dW is written once,
// in FP32 sums whose order is that of the tokens (deterministic; the only atomics
// are integer counts):
//   1. embed_sort: each workgroup owns a range of rows and reads all ids (they stay
//      in L2).  It counts the ids below its range, which is where its tokens go in
//      the sorted order, without waiting for another workgroup, and per wave and
//      row the ids of its range; then every wave places its share of the tokens in
//      their order, ranking equal ids by comparing bits across the lanes.
//   2. embed_walk: a workgroup walks the sorted tokens of 16 positions, eight rows of
//      dY in flight, and writes a row of dW where its run of tokens ends; runs of
//      more than kEmbedPart tokens (a token that is a tenth of a text would keep one
//      workgroup busy long after the others) leave FP32 partial rows.  Other workgroups
//      of the launch write the zeros of the rows without a token.
//   3. embed_join adds the partial rows of the long runs, in order.
// Few tokens and a small table: embed_scan does it in one launch, a workgroup per row
// that looks for its tokens itself.

#include "packed.hpp"

#include "common.hpp"

namespace lt {
namespace {

constexpr int kThreads = 256;

// tpr threads per token row (a power of two), kThreads / tpr rows per workgroup.  4096 rows
// of 4096 10 us (6.9 TB/s; the rows partly from cache), 8191 rows of 5120 25 us (6.6).
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

// ------------------------------------------------------------ 1: sort
constexpr int kSortWaves = 16;
constexpr int kSortMaxRows = 1024;
constexpr int kIdBatches = 8;          // 64-id batches a wave loads together

// range: rows v0 .. v0 + R - 1, R = 1 << bits.  Latency-bound: two passes over the ids,
// 4096 of them in 7 us, 8191 in 12.5.
__global__ void __launch_bounds__(64 * kSortWaves)
embed_sort_kernel(const int64_t* __restrict__ ids, int64_t T, int64_t V, int bits, int32_t* __restrict__ start,
                  int32_t* __restrict__ tokens) {
  __shared__ int at[kSortWaves][kSortMaxRows];     // per wave and row: count, then next position
  __shared__ int below_s[kSortWaves], sum_s[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int R = 1 << bits;
  const int64_t v0 = (int64_t)blockIdx.x << bits;
  for (int i = tid; i < kSortWaves * R; i += 64 * kSortWaves) at[i >> bits][i & (R - 1)] = 0;
  __syncthreads();

  // the wave's 64-id batches
  const int64_t nb = (T + 63) / 64, per = (nb + kSortWaves - 1) / kSortWaves;
  const int64_t b0 = wave * per, b1 = b0 + per < nb ? b0 + per : nb;
  auto each = [&](auto f) {
    for (int64_t b = b0; b < b1; b += kIdBatches) {
      int64_t id[kIdBatches];
#pragma unroll
      for (int u = 0; u < kIdBatches; ++u) {
        const int64_t t = (b + u) * 64 + lane;
        id[u] = b + u < b1 && t < T ? ids[t] : -1;
      }
#pragma unroll
      for (int u = 0; u < kIdBatches; ++u) f((b + u) * 64 + lane, id[u]);
    }
  };
  int below = 0;
  each([&](int64_t, int64_t id) {
    if (id >= 0 && id < V) {
      if (id < v0) ++below;
      else if (id < v0 + R) atomicAdd(&at[wave][(int)(id - v0)], 1);
    }
  });
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) below += __shfl_xor(below, m);
  if (lane == 0) below_s[wave] = below;
  __syncthreads();

  // thread = row: its total, the sum of the totals before it
  int total = 0;
  if (tid < R)
    for (int w = 0; w < kSortWaves; ++w) total += at[w][tid];
  int scan = total;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int v = __shfl_up(scan, m);
    if (lane >= m) scan += v;
  }
  if (lane == 63) sum_s[wave] = scan;
  __syncthreads();
  int pos = scan - total;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    pos += below_s[w];
    if (w < wave) pos += sum_s[w];
  }
  if (tid < R) {
    if (v0 + tid < V) start[v0 + tid] = pos;
    if (v0 + tid == V - 1) start[V] = pos + total;
    for (int w = 0; w < kSortWaves; ++w) {
      const int n = at[w][tid];
      at[w][tid] = pos;
      pos += n;
    }
  }
  __syncthreads();

  each([&](int64_t t, int64_t id) {
    const bool mine = id >= v0 && id < v0 + R && id < V;
    uint64_t peers = __builtin_amdgcn_ballot_w64(mine);
    if (peers == 0) return;
    const int l = mine ? (int)(id - v0) : 0;
    for (int b = 0; b < bits; ++b) {
      const bool on = (l >> b) & 1;
      const uint64_t bal = __builtin_amdgcn_ballot_w64(on);
      peers &= on ? bal : ~bal;
    }
    if (mine) {
      const int rank = __popcll(peers & ((1ull << lane) - 1));
      const int p = at[wave][l];
      tokens[p + rank] = (int32_t)t;
      if (rank == 0) at[wave][l] = p + __popcll(peers);
    }
  });
}

// ------------------------------------------------------------ 2: walk
__device__ __forceinline__ void store_row(const EmbedBwdArgs& a, int64_t v, int64_t col, const float (&acc)[8]) {
  lt_half* dst = a.dW + v * a.lddw + col;
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

constexpr int kRowWaves = kThreads / 64;

// partial row of piece k (sorted positions p = s + k kEmbedPart ...) of a long run: the last
// piece of one run and the first of the next can start in the same window of positions
__device__ __forceinline__ int64_t part_row(int p, int k) { return 2 * (int64_t)(p / kEmbedPart) + (k == 0); }

// Workgroups 0 .. parts x ncb - 1: (kEmbedPart positions, 2048 columns).  They take the
// runs, and the pieces of long runs, that start in their positions: at most
// 2 kEmbedPart - 1 tokens.  The others: 2^zbits lanes a row (up to a wave), zeros where no token
// falls (non-temporal, so that they do not evict the tokens' rows; more rows a wave: level).
// Bound by the writes of dW: 32000 x 4096 (262 MB) and 4096 tokens in 42 us, 152064 x 5120
// (1557 MB) and 8191 tokens in 281 us (5.8 TB/s).
__global__ void __launch_bounds__(kThreads)
embed_walk_kernel(const EmbedBwdArgs a, int parts, int ncb, int zbits) {
  constexpr int C = kEmbedPart;
  static_assert(2 * C <= 64, "a lane per token");
  const int lane = threadIdx.x & 63;
  if (blockIdx.x >= (unsigned)(parts * ncb)) {
    const int64_t v = (int64_t)(blockIdx.x - parts * ncb) * (kThreads >> zbits) + (threadIdx.x >> zbits);
    if (v >= a.V || a.start[v] != a.start[v + 1]) return;
    for (int64_t col = (threadIdx.x & ((1 << zbits) - 1)) * 8; col < a.H; col += 8 << zbits)
      __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4*>(a.dW + v * a.lddw + col));
    return;
  }
  const int n = a.start[a.V];
  const int p0 = (int)(blockIdx.x / ncb) * C;
  const int64_t col = ((int64_t)(blockIdx.x % ncb) * kThreads + threadIdx.x) * 8;
  // lane = position p0 + lane: its token and row, whether its piece starts here,
  // whether it is the piece's last
  int t = 0, v = 0, row = 0;
  bool mine = false, last = false, whole = false;
  if (lane < 2 * C && p0 + lane < n) {
    const int p = p0 + lane;
    t = a.tokens[p];
    v = (int)a.ids[t];
    const int s = a.start[v], e = a.start[v + 1];
    whole = e - s <= C;
    const int k = whole ? 0 : (p - s) / C;
    const int ps = s + k * C;                        // the piece's first position
    mine = ps >= p0 && ps < p0 + C;
    last = p + 1 == (whole ? e : min(ps + C, e));
    row = (int)part_row(ps, k);
  }
  const uint64_t mines = __builtin_amdgcn_ballot_w64(mine);
  const uint64_t lasts = __builtin_amdgcn_ballot_w64(last), wholes = __builtin_amdgcn_ballot_w64(whole);
  const bool in = col < a.H;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma nounroll
  for (int i0 = 0; i0 < 2 * C; i0 += 8) {
    if (!(mines >> i0 & 0xff)) continue;
    half8 g[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t tu = __builtin_amdgcn_readlane(t, i0 + u);
      g[u] = as_half8(in && (mines >> (i0 + u) & 1) ? ld16(a.dY + tu * a.lddy + col) : u32x4{0, 0, 0, 0});
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u;
      if (!(mines >> i & 1)) continue;               // uniform, as all that follows
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += (float)g[u][e];
      if (!(lasts >> i & 1)) continue;
      if (in) {
        if (wholes >> i & 1) {
          store_row(a, __builtin_amdgcn_readlane(v, i), col, acc);
        } else {
          float* dst = a.part + (int64_t)__builtin_amdgcn_readlane(row, i) * a.H + col;
          *reinterpret_cast<float4*>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
          *reinterpret_cast<float4*>(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    }
  }
}

// ------------------------------------------------------------ 3: join
// Workgroup = (kJoinSpan windows of kEmbedPart positions, 256 columns), for the long runs
// that start there (a window holds the start of one at most, and its last token is of
// that run).  Each of 8 thread groups adds an eighth of the partial rows, eight loads
// in flight, then the groups' sums are added, all in order.  Bound by latency and by the
// longest run, hence the narrow columns: the gradient of 16384 tokens of 32000 x 4096 takes
// 78 us, with half of the tokens the same 100, all 131 (one group of four waves per 512 columns:
// 107 and 156); a window a workgroup costs ordinary texts 3 us, four 4.
constexpr int kJoinSpan = 2;
constexpr int kJoinLanes = 32, kJoinGroups = kThreads / kJoinLanes;
__global__ void __launch_bounds__(kThreads)
embed_join_kernel(const EmbedBwdArgs a) {
  constexpr int C = kEmbedPart;
  __shared__ float red[kJoinGroups][kJoinLanes * 8];
  const int lane = threadIdx.x & 63, grp = threadIdx.x / kJoinLanes, c = threadIdx.x % kJoinLanes;
  const int n = a.start[a.V];
  // lane = window
  int v = 0, s = 0, e = 0;
  bool mine = false;
  const int p0 = ((int)blockIdx.x * kJoinSpan + lane) * C;
  if (lane < kJoinSpan && p0 < n) {
    v = (int)a.ids[a.tokens[min(p0 + C, n) - 1]];
    s = a.start[v];
    e = a.start[v + 1];
    mine = e - s > C && s >= p0;
  }
  uint64_t runs = __builtin_amdgcn_ballot_w64(mine);           // the same in every wave
  const int64_t col = ((int64_t)blockIdx.y * kJoinLanes + c) * 8;
  const bool in = col < a.H;
  for (; runs != 0; runs &= runs - 1) {
    const int w = __builtin_ctzll(runs);
    const int sw = __builtin_amdgcn_readlane(s, w), ew = __builtin_amdgcn_readlane(e, w);
    const int pieces = (ew - sw + C - 1) / C, per = (pieces + kJoinGroups - 1) / kJoinGroups;
    const int k0 = grp * per, k1 = min(k0 + per, pieces);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = k0; k < k1; k += 8) {
      float4 x[8], y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float* src = a.part + part_row(sw + (k + u) * C, k + u) * a.H + col;
        const bool ok = in && k + u < k1;
        x[u] = ok ? *reinterpret_cast<const float4*>(src) : make_float4(0.f, 0.f, 0.f, 0.f);
        y[u] = ok ? *reinterpret_cast<const float4*>(src + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        acc[0] += x[u].x; acc[1] += x[u].y; acc[2] += x[u].z; acc[3] += x[u].w;
        acc[4] += y[u].x; acc[5] += y[u].y; acc[6] += y[u].z; acc[7] += y[u].w;
      }
    }
    __syncthreads();                                 // red is free
#pragma unroll
    for (int q = 0; q < 8; ++q) red[grp][c * 8 + q] = acc[q];
    __syncthreads();
    if (grp == 0 && in) {
      for (int r = 1; r < kJoinGroups; ++r)
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] += red[r][c * 8 + q];
      store_row(a, __builtin_amdgcn_readlane(v, w), col, acc);
    }
  }
}

// ------------------------------------------------------------ few tokens: scan
// One workgroup per (row of the table, 2048 columns), up to kThreads tokens.
__global__ void __launch_bounds__(kThreads)
embed_scan_kernel(const EmbedBwdArgs a) {
  __shared__ int hits[kThreads];
  __shared__ int counts[kRowWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t v = blockIdx.x;
  const int64_t col = ((int64_t)blockIdx.y * kThreads + tid) * 8;
  const bool hit = tid < a.T && a.ids[tid] == v;
  const uint64_t bal = __builtin_amdgcn_ballot_w64(hit);
  if (lane == 0) counts[wave] = __popcll(bal);
  __syncthreads();
  int at = 0, n = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) at += counts[w];
    n += counts[w];
  }
  if (hit) hits[at + __popcll(bal & ((1ull << lane) - 1))] = tid;
  __syncthreads();
  if (col >= a.H || (a.accumulate && n == 0)) return;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < n; k += 4) {
    half8 g[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      g[u] = as_half8(k + u < n ? ld16(a.dY + (int64_t)hits[k + u] * a.lddy + col) : u32x4{0, 0, 0, 0});
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += (float)g[u][e];
  }
  store_row(a, v, col, acc);
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

// One launch pays while a workgroup per row costs less than three launches: one step
// of up to 256 ids, and rows for a few rounds of workgroups.  us, scanning / sorted:
// 256 tokens of 4000 x 256: 4.5 / 12; of 32000 x 256: 15.5 / 16.4, accumulating 11.9 /
// 15.2; of 32000 x 4096 (two column blocks): 46 / 41, accumulating 22 / 17.
constexpr int64_t kScanRows = 32768;

hipError_t embed_bwd_launch(const EmbedBwdArgs& a, hipStream_t s) {
  const int wide = (int)((a.H + kThreads * 8 - 1) / (kThreads * 8));   // 2048-column blocks
  if (a.T <= kThreads && a.V * wide <= kScanRows) {
    hipLaunchKernelGGL(embed_scan_kernel, dim3((unsigned)a.V, (unsigned)wide), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  }
  int bits = 0;
  while ((1 << bits) < embed_sort_rows(a.V)) ++bits;
  hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)((a.V + (1 << bits) - 1) >> bits)), dim3(64 * kSortWaves), 0, s,
                     a.ids, a.T, a.V, bits, a.start, a.tokens);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int parts = (int)embed_parts(a.T);
  int zbits = 0;
  while (zbits < 6 && (8 << zbits) < a.H) ++zbits;
  const int64_t per = kThreads >> zbits, rows = a.accumulate ? 0 : (a.V + per - 1) / per;
  hipLaunchKernelGGL(embed_walk_kernel, dim3((unsigned)(parts * wide + rows)), dim3(kThreads), 0, s, a, parts, wide,
                     zbits);
  if ((e = hipGetLastError()) != hipSuccess || a.T <= kEmbedPart) return e;
  hipLaunchKernelGGL(embed_join_kernel,
                     dim3((unsigned)((parts + kJoinSpan - 1) / kJoinSpan),
                     (unsigned)((a.H / 8 + kJoinLanes - 1) / kJoinLanes)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace lt
