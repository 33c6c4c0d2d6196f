// The projection for a few rows (decoding), and the contraction of the rows with their adapters.
//
// linear_small: y[t][j] = sum_i x[t][i] W[j][i], up to 16 rows.  Bound: memory, half a byte a weight, but at a few
// megabytes the time is a chain of latencies: the launch, the loads, the products, one exchange, the store.  With
// W = z0 + Delta k a group of input channels contributes  Delta sum k x + z0 sum x, so the tensor cores multiply the
// codes themselves: 0x4180 | k << 3 is the bf16 number 16 + k, two codes leave a packed word per shift and mask, and
//   y = sum over groups of  Delta (sum (16 + k) x) + (z0 - 16 Delta) sum x
// in fp32, without a rounding of any weight.  (The offset is the smallest whose sums with every code lie between two powers
// of two, so that the code is a field of the number; it costs 4 of the 24 bits of the fp32 sums.)
// A CTA owns 16 (or 32) output channels.  Asynchronous copies bring a slice of the rows, the codes and the grid to shared
// memory, all of a layer of 4096 input channels at once; sixteen warps split the slice and their sums meet at the end.
// Channels are taken in an order that lets a thread read 16 of them from consecutive addresses for the codes and for x
// alike: a product over them does not ask for their order.  h comes from a launch of its own, which this one overlaps up
// to its last step; the adapters' output sides are copied meanwhile.
// The code is kept short (rolled loops, no divisions): it runs once a launch from cold instruction caches.  With the same
// work unrolled and its loads in registers a CTA took 14000 cycles; with clusters of eight CTAs that form h themselves
// and split the input channels it took 12700, and such a launch does not overlap the one before it.
//
// shrink: h[t][r] = scale_a sum_i x[t][i] in_a[r][i].  Bound: memory, one pass over the rows and over the adapters in
// use.  Three forms: a CTA for each row and two ranks for few rows, tiles of 16 or 32 rows on mma.sync for more, where
// the passes over a tile are one per distinct adapter in it, and for many the tiles of shrink_tc.cu.
#include <cooperative_groups.h>

#include "adapt.h"

namespace cg = cooperative_groups;

namespace admmq {
namespace {

constexpr int THREADS = 256, WARPS = 8;          // of the contractions with the adapters

// ------------------------------------------------------------------ few rows: the projection
struct SmallParams {
  PackedLayer L;
  const bf16* x;
  long long ldx;
  bf16* y;
  long long ldy;
  int T;
  int slice;                      // blocks of 64 input channels in shared memory at once
  uint32_t group_inv;             // ceil(2^32 / blocks of a group); 1: a block is a group, 0: one group
  int x_stride;                   // elements of a copied row
  int warps_log, out_log;         // 2^warps_log warps copy a row, 2^out_log lanes finish an output
  int at_grid, at_x, at_sx, at_up;   // bytes: after the codes, the grid, the rows, the sums of x
  const bf16* up;                 // adapters' output side [n][rank][d_out], NULL: none
  const int* row_adapter;
  const float* h;                 // [T][rank]
  int n_adapters, rank;
  bool up_copied;                 // the output sides fit in shared memory
};

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float s) {
  const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 x = bf16x2_to_float2(av[e]), y = bf16x2_to_float2(bv[e]);
    s = fmaf(x.x, y.x, fmaf(x.y, y.y, s));
  }
  return s;
}

constexpr int MAIN_WARPS = 16, MAIN_THREADS = 32 * MAIN_WARPS;
constexpr int SLICE_MAX = 64;                        // blocks of 64 input channels in shared memory
constexpr int X_BYTES_MAX = 132 * 1024;              // bytes of rows in shared memory
constexpr int UP_MAX = 128;                          // rows * rank up to which the output sides are copied

__device__ __forceinline__ void copy16(void* dst, const void* src, bool in) {      // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(in ? 16 : 0)
               : "memory");
}

// MT tiles of 16 channels, NT tiles of 8 rows.  Shared memory: codes [block][channel][32 bytes], grid [block][channel], rows
// [T][x_stride], sums of x [block][T], output sides [row][rank][channel]; at the end the warps' sums over the codes.
template <int MT, int NT>
__global__ void __launch_bounds__(MAIN_THREADS, MT* NT == 1 ? 2 : 1) linear_small_kernel(const __grid_constant__ SmallParams P) {
  constexpr int CH = 16 * MT, ROWS = 8 * NT;
  extern __shared__ __align__(16) uint8_t work[];
  __shared__ int own[ROWS];                                            // adapters of the rows, -1: none
  bf16* x_s = reinterpret_cast<bf16*>(work + P.at_x);
  float* sx = reinterpret_cast<float*>(work + P.at_sx);
  bf16* up_s = reinterpret_cast<bf16*>(work + P.at_up);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, q = lane & 3;
  const int j0 = (int)blockIdx.x * CH;
  const int p = P.L.d_out, n = P.L.d_in, T = P.T, rank = P.rank;
  const int rows_in = min(CH, p - j0);                                 // output channels of the tile
  if (tid < ROWS) own[tid] = P.up != nullptr && tid < T ? row_adapter_of(P.row_adapter, tid, P.n_adapters) : -1;
  // rows to warps, 2^warps_log to a row
  const int my_row = warp >> P.warps_log, lanes = 32 << P.warps_log, my_lane = tid & (lanes - 1);

  float y[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) y[m][t][e] = 0.0f;

#pragma unroll 1
  for (int ibA = 0; ibA < P.L.nib; ibA += P.slice) {
  const int nb = min(P.slice, P.L.nib - ibA);
  if (ibA > 0) __syncthreads();                                        // the slice before is used up
  // ---- everything of the slice is asked for at once: rows, codes, grid
  if (my_row < T)
#pragma unroll 1
    for (int c = my_lane * 8; c < nb * CODE_BLOCK; c += lanes * 8) {
      const int i = ibA * CODE_BLOCK + c;
      copy16(x_s + my_row * P.x_stride + c, P.x + my_row * P.ldx + (i < n ? i : 0), i < n);
    }
  asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll 1
  for (int c = tid; c < nb * CH * 2; c += MAIN_THREADS) {              // 16 bytes: half a channel's block
    const int b = c / (CH * 2), k = c % (CH * 2);
    const bool in = (k >> 1) < rows_in;
    copy16(work + c * 16, P.L.codes + (in ? ((long long)(ibA + b) * p + j0) * BLOCK_WORDS + k * 4 : 0), in);
  }
#pragma unroll 1
  for (int c = tid; c < nb * (CH / 2); c += MAIN_THREADS) {            // 16 bytes: two channels' pairs
    const int b = c / (CH / 2), k = c % (CH / 2);
    const bool in = 2 * k < rows_in;                                   // d_out is a multiple of 8
    const int ib = ibA + b, grp = P.group_inv > 1 ? (int)__umulhi((uint32_t)ib, P.group_inv) : P.group_inv ? ib : 0;
    copy16(work + P.at_grid + c * 16, P.L.grid + (in ? (long long)grp * p + j0 + 2 * k : 0), in);
  }
  if (P.up_copied && ibA == 0) {
#pragma unroll 1
    for (int o = warp; o < T * rank; o += MAIN_WARPS) {                // a (row, rank) a warp, 8 channels a lane
      const int t = o / rank, r = o - t * rank, a = row_adapter_of(P.row_adapter, t, P.n_adapters);
      if (lane < CH / 8) {
        const bool in = a >= 0 && lane * 8 < rows_in;
        copy16(up_s + o * CH + lane * 8, P.up + (in ? ((long long)a * rank + r) * p + j0 + lane * 8 : 0), in);
      }
    }
  }
  asm volatile("cp.async.commit_group;\ncp.async.wait_group 1;" ::: "memory");
  __syncthreads();                                 // the rows are in place: their sums over blocks, 8 threads a block
  if (my_row < T)
#pragma unroll 2
    for (int c = my_lane; c < nb * 8; c += lanes) {                    // (nb 8 is a multiple of 8: whole groups of lanes)
      const uint32_t one = 0x3f803f80u, mask = 0xffu << (lane & 24);
      float f = dot8(*reinterpret_cast<const uint4*>(x_s + my_row * P.x_stride + c * 8), make_uint4(one, one, one, one), 0.0f);
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) f += __shfl_xor_sync(mask, f, d);
      if ((c & 7) == 0) sx[(c >> 3) * T + my_row] = f;
    }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();

  // ---- products, block by block
  const int b0 = nb * warp / MAIN_WARPS;
  const uint2* cs = reinterpret_cast<const uint2*>(work) + (b0 * CH + g) * 4 + q;
  const float2* gs = reinterpret_cast<const float2*>(work + P.at_grid) + b0 * CH + g;
  const bf16* xp = x_s + g * P.x_stride + b0 * CODE_BLOCK + 16 * q;
  const float* sp = sx + b0 * T + 2 * q;
#pragma unroll 1
  for (int b = nb * (warp + 1) / MAIN_WARPS - b0; b > 0; --b) {
    float acc[MT][NT][4];
    uint4 xv[NT][2];
    uint2 c[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) c[m][hh] = cs[(16 * m + 8 * hh) * 4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      xv[t][0] = xv[t][1] = make_uint4(0, 0, 0, 0);
      if (8 * t + g < T) {
        xv[t][0] = *reinterpret_cast<const uint4*>(xp + 8 * t * P.x_stride);
        xv[t][1] = *reinterpret_cast<const uint4*>(xp + 8 * t * P.x_stride + 8);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][t][e] = 0.0f;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)                    // 8 channels of this thread
#pragma unroll
      for (int s = 0; s < 2; ++s)                  // pairs 2 s and 2 s + 1 of the word
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t c0 = w == 0 ? c[m][0].x : c[m][0].y, c1 = w == 0 ? c[m][1].x : c[m][1].y;
          const uint32_t a[4] = {((s == 0 ? c0 << 3 : c0 >> 5) & 0x00780078u) | 0x41804180u,
                                 ((s == 0 ? c1 << 3 : c1 >> 5) & 0x00780078u) | 0x41804180u,
                                 ((c0 >> (8 * s + 1)) & 0x00780078u) | 0x41804180u,
                                 ((c1 >> (8 * s + 1)) & 0x00780078u) | 0x41804180u};
#pragma unroll
          for (int t = 0; t < NT; ++t)
            mma_bf16(acc[m][t], a, s == 0 ? xv[t][w].x : xv[t][w].z, s == 0 ? xv[t][w].y : xv[t][w].w);
        }
    // the block's share of y; s0, s1: sums of x of the rows 8 t + 2 q and the next
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float s0 = 8 * t + 2 * q < T ? sp[8 * t] : 0.0f, s1 = 8 * t + 2 * q + 1 < T ? sp[8 * t + 1] : 0.0f;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const float2 g0 = gs[16 * m], g1 = gs[16 * m + 8];
        const float z0 = fmaf(-16.0f, g0.x, g0.y), z1 = fmaf(-16.0f, g1.x, g1.y);
        y[m][t][0] = fmaf(g0.x, acc[m][t][0], fmaf(z0, s0, y[m][t][0]));
        y[m][t][1] = fmaf(g0.x, acc[m][t][1], fmaf(z0, s1, y[m][t][1]));
        y[m][t][2] = fmaf(g1.x, acc[m][t][2], fmaf(z1, s0, y[m][t][2]));
        y[m][t][3] = fmaf(g1.x, acc[m][t][3], fmaf(z1, s1, y[m][t][3]));
      }
    }
    cs += CH * 4;
    gs += CH;
    xp += CODE_BLOCK;
    sp += T;
  }
  }
  __syncthreads();
  float* red = reinterpret_cast<float*>(work);     // [row][channel][17 warps]
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float* o = red + ((8 * t + 2 * q) * CH + 16 * m + g) * (MAIN_WARPS + 1) + warp;
      o[0] = y[m][t][0];
      o[CH * (MAIN_WARPS + 1)] = y[m][t][1];
      o[8 * (MAIN_WARPS + 1)] = y[m][t][2];
      o[(CH + 8) * (MAIN_WARPS + 1)] = y[m][t][3];
    }
  __syncthreads();
  if (P.up != nullptr) pdl_wait();                 // h is complete from here on
  // ---- 2^out_log lanes an output, the warps' sums and the ranks shared out among them
  const int lanes_out = 1 << P.out_log, sub = lane & (lanes_out - 1);
#pragma unroll 1
  for (int o = tid >> P.out_log; o < T * CH; o += MAIN_THREADS >> P.out_log) {
    const int t = o / CH, c = o % CH, a = own[t];
    float v = 0.0f;
#pragma unroll 4
    for (int w = sub; w < MAIN_WARPS; w += lanes_out) v += red[o * (MAIN_WARPS + 1) + w];
    if (a >= 0 && c < rows_in) {
      const bf16* up = P.up_copied ? up_s + t * rank * CH + c : P.up + (long long)a * rank * p + j0 + c;
      const long long ld = P.up_copied ? CH : p;
#pragma unroll 4
      for (int r = sub; r < rank; r += lanes_out) v = fmaf(P.h[t * rank + r], __bfloat162float(up[r * ld]), v);
    }
    const uint32_t mask = lanes_out == 32 ? 0xffffffffu : ((1u << lanes_out) - 1u) << (lane & -lanes_out);
#pragma unroll 1
    for (int d = lanes_out >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(mask, v, d);
    if (sub == 0 && c < rows_in) P.y[t * P.ldy + j0 + c] = __float2bfloat16_rn(v);
  }
}

// ------------------------------------------------------------------ rows times adapters
struct ShrinkParams {
  const bf16* x;
  long long ldx, T;
  int K;
  const bf16* mat;                // [n][rank][K]
  const float* scale;
  int n, rank;
  const int* row_adapter;
  float* h;                       // [T][rank]
};

// One row and two ranks a CTA, four warps a rank: 4096 channels are four loads of a thread for the row and four for the
// adapter, all under way at once.  (A warp a rank made four rounds of them, 5.2 us for one row, and the projection's last
// step waits for it.)
__global__ void __launch_bounds__(THREADS) shrink_rows_kernel(const __grid_constant__ ShrinkParams P) {
  pdl_launch();
  __shared__ float part[WARPS];
  const long long t = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = warp >> 2;
  const int r = blockIdx.y * 2 + half, first = (threadIdx.x & 127) * 8;
  const bf16* x = P.x + t * P.ldx;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const int a = row_adapter_of(P.row_adapter, t, P.n);
  const bf16* m = P.mat + ((long long)(a < 0 ? 0 : a) * P.rank + r) * P.K;
  float v = 0.0f;
#pragma unroll 1
  for (int i = first; i < P.K; i += 4 * 1024) {
    uint4 xv[4], mv[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) xv[u] = i + 1024 * u < P.K ? __ldg(reinterpret_cast<const uint4*>(x + i + 1024 * u)) : zero;
#pragma unroll
    for (int u = 0; u < 4; ++u) mv[u] = i + 1024 * u < P.K ? __ldg(reinterpret_cast<const uint4*>(m + i + 1024 * u)) : zero;
#pragma unroll
    for (int u = 0; u < 4; ++u) v = dot8(xv[u], mv[u], v);
  }
  v = warp_sum(v);
  if (lane == 0) part[warp] = v;
  __syncthreads();
  if (threadIdx.x < 2) {
    const float* s = part + 4 * threadIdx.x;
    P.h[t * P.rank + blockIdx.y * 2 + threadIdx.x] = a >= 0 ? ((s[0] + s[1]) + (s[2] + s[3])) * P.scale[a] : 0.0f;
  }
}

// Tiles of 16 MT rows and 8 NT ranks.  A cluster shares a tile: its CTAs, and the warps in them, split the contracted
// channels, 32 of them a step; the CTAs' sums meet over distributed shared memory, in rank order.
template <int MT, int NT>
__global__ void __launch_bounds__(THREADS, MT * NT <= 4 ? 2 : 1) shrink_tile_kernel(const __grid_constant__ ShrinkParams P) {
  pdl_launch();
  constexpr int TM = 16 * MT, RN = 8 * NT;
  extern __shared__ float red[];                   // [WARPS][TM][RN], then this CTA's sums [TM][RN]
  float* part = red + WARPS * TM * RN;
  __shared__ int own[TM];
  cg::cluster_group cluster = cg::this_cluster();
  const int share = (int)cluster.block_rank(), shares = (int)cluster.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, q = lane & 3;
  const long long t0 = (long long)(blockIdx.x / shares) * TM;
  if (threadIdx.x < TM) own[threadIdx.x] = t0 + threadIdx.x < P.T ? row_adapter_of(P.row_adapter, t0 + threadIdx.x, P.n) : -1;
  const bf16* xr[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const long long t = t0 + 16 * m + 8 * hh + g;
      xr[m][hh] = P.x + (t < P.T ? t : P.T - 1) * P.ldx;      // rows past the end: any row, their results are dropped
    }
  __syncthreads();
  for (int last = -1;;) {
    int a = 0x7fffffff;                            // the next adapter of this tile, in rising order
    for (int t = lane; t < TM; t += 32) a = own[t] > last ? min(a, own[t]) : a;
    a = __reduce_min_sync(0xffffffffu, a);
    if (a == 0x7fffffff) break;
    last = a;
    float acc[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int nn = 0; nn < NT; ++nn)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][nn][e] = 0.0f;
    const bf16* mat = P.mat + (long long)a * P.rank * P.K;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    constexpr int UNR = 2 * MT + NT <= 4 ? 4 : 2 * MT + NT <= 8 ? 2 : 1;
    const int chunk = 32 * UNR, stride = WARPS * chunk * shares;     // a warp's neighbouring channels fill cache lines
    for (int k0 = (share * WARPS + warp) * chunk; k0 < P.K; k0 += stride) {
      uint4 av[UNR][MT][2], bv[UNR][NT];
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        const int i = k0 + 32 * u + 8 * q;
        const bool in = i < P.K;                   // K is a multiple of 8
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            av[u][m][hh] = in ? __ldg(reinterpret_cast<const uint4*>(xr[m][hh] + i)) : zero;
#pragma unroll
        for (int nn = 0; nn < NT; ++nn)
          bv[u][nn] = in && 8 * nn + g < P.rank
                          ? __ldg(reinterpret_cast<const uint4*>(mat + (long long)(8 * nn + g) * P.K + i)) : zero;
      }
#pragma unroll
      for (int u = 0; u < UNR; ++u)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint4 &lo = av[u][m][0], &hi = av[u][m][1];
          const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
          for (int nn = 0; nn < NT; ++nn) {
            mma_bf16(acc[m][nn], a0, bv[u][nn].x, bv[u][nn].y);
            mma_bf16(acc[m][nn], a1, bv[u][nn].z, bv[u][nn].w);
          }
        }
    }
    // a row has one adapter: its sums go straight to their place
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
        if (own[16 * m + 8 * hh + g] == a) {
          float* o = red + ((long long)warp * TM + 16 * m + 8 * hh + g) * RN + 2 * q;
#pragma unroll
          for (int nn = 0; nn < NT; ++nn)
            *reinterpret_cast<float2*>(o + 8 * nn) = make_float2(acc[m][nn][2 * hh], acc[m][nn][2 * hh + 1]);
        }
  }
  __syncthreads();
  for (int o = threadIdx.x; o < TM * RN; o += THREADS) {
    if (own[o / RN] < 0) continue;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) v += red[w * TM * RN + o];
    part[o] = v;
  }
  cluster.sync();
  for (int o = share * THREADS + threadIdx.x; o < TM * RN; o += shares * THREADS) {
    const int t = o / RN, r = o % RN;
    if (t0 + t >= P.T || r >= P.rank) continue;
    float v = 0.0f;
    if (own[t] >= 0) {
      for (int k = 0; k < shares; ++k) v += cluster.map_shared_rank(part, k)[o];
      v *= P.scale[own[t]];
    }
    P.h[(t0 + t) * P.rank + r] = v;
  }
  cluster.sync();                                  // no CTA leaves while its sums are read
}

template <int MT, int NT>
cudaError_t launch_tile(const ShrinkParams& P, int sms, int spare, cudaStream_t stream) {
  constexpr int BYTES = (WARPS + 1) * 16 * MT * 8 * NT * 4;
  const cudaError_t e = ensure_dynamic_smem((const void*)shrink_tile_kernel<MT, NT>, BYTES);
  if (e != cudaSuccess) return e;
  const long long tiles = (P.T + 16 * MT - 1) / (16 * MT);
  // CTAs of a tile: as many as run at once with two on every multiprocessor and leave each at least two steps of all its
  // warps (8192 rows of 12288, rank 16: 21.7 us in one turn, 25.6 in the two of twice as many CTAs)
  int shares = 1;
  while (shares < 8 && tiles * 2 * shares <= 2 * sms && P.K >= 2 * WARPS * 32 * 2 * shares) shares *= 2;
  // Half as many, if the multiprocessors that the projection after this launch leaves then suffice: it starts at once, and
  // needs the results for its last steps only (4096 -> 12288, both launches: 203 rows of 24 adapters 49.0 -> 44.9 us, 150
  // rows of 60 57.2 -> 46.1).
  if (tiles * shares > spare && shares > 1 && tiles * (shares / 2) <= spare) shares /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * shares));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = shares;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, shrink_tile_kernel<MT, NT>, P);
}

template <int MT, int NT>
cudaError_t launch_small(SmallParams& P, cudaStream_t stream) {
  constexpr int CH = 16 * MT, RED = 8 * NT * CH * (MAIN_WARPS + 1) * 4;
  P.slice = P.L.nib < SLICE_MAX ? P.L.nib : SLICE_MAX;
  while (P.T * P.slice * CODE_BLOCK * 2 > X_BYTES_MAX) P.slice = (P.slice + 1) / 2;
  const int group = P.L.gs == P.L.d_in ? 0 : P.L.gs / CODE_BLOCK;
  P.group_inv = group <= 1 ? (uint32_t)group : (uint32_t)(((1ULL << 32) + group - 1) / group);
  P.x_stride = P.slice * CODE_BLOCK + 8;
  while (P.T << (P.warps_log + 1) <= MAIN_WARPS) ++P.warps_log;
  while (P.out_log < 4 && P.T * CH << (P.out_log + 1) <= MAIN_THREADS) ++P.out_log;
  P.at_grid = P.slice * CH * 32;
  P.at_x = P.at_grid + P.slice * CH * 8;
  P.at_sx = P.at_x + P.T * P.x_stride * 2;
  const int after = (P.at_sx + P.T * P.slice * 4 + 15) / 16 * 16;
  P.at_up = after > RED ? after : RED;
  P.up_copied = P.up != nullptr && P.T * P.rank <= UP_MAX;
  const int bytes = P.at_up + (P.up_copied ? P.T * P.rank * CH * 2 : 0);
  const cudaError_t e = ensure_dynamic_smem((const void*)linear_small_kernel<MT, NT>, bytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((P.L.d_out + CH - 1) / CH);
  cfg.blockDim = dim3(MAIN_THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = P.up != nullptr ? 1 : 0;          // with adapters it may start beside the shrink launch before it
  return cudaLaunchKernelEx(&cfg, linear_small_kernel<MT, NT>, P);
}

constexpr long long SHRINK_ROWS_MAX = 64;

}  // namespace

cudaError_t launch_shrink(const bf16* x, long long ldx, long long T, int K, const AdapterView& ad,
                          const int* row_adapter, float* h, int spare, int* status, cudaStream_t stream) {
  const ShrinkParams P = {x, ldx, T, K, ad.in, ad.scale, ad.n, ad.rank, row_adapter, h};
  if (T <= SHRINK_ROWS_MAX) {
    shrink_rows_kernel<<<dim3((unsigned)T, ad.rank / 2), THREADS, 0, stream>>>(P);
    return cudaGetLastError();
  }
  // On the tensor cores' tiles a row costs the same at any rank, here it costs the adapters' rows again for every 16 or 32
  // of the rows.  K = 4096: rank 16, 2048 rows 8.4 us here, 10.8 there, 16384 rows 32 and 31 (K = 12288: 6011 rows 56 and
  // 37); rank 32, 520 rows 7.5 and 9.7, 1100 rows 17.6 and 10.8; rank 128, 200 rows 12.3 and 14.5, 520 rows 26 and 15.
  if (ad.rank > 16 ? T * ad.rank >= 32768 : T > 4096)
    return launch_shrink_tc(x, ldx, T, K, ad, row_adapter, h, status, stream);
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  // Tiles of 32 rows read the adapters half as often; tiles of 16 meet fewer distinct adapters and are more.
  if (T > 1024) {                                // (rank 24 has up to 1365 rows here)
    if (ad.rank <= 8) return launch_tile<2, 1>(P, sms, spare, stream);
    if (ad.rank <= 16) return launch_tile<2, 2>(P, sms, spare, stream);
  }
  if (ad.rank <= 8) return launch_tile<1, 1>(P, sms, spare, stream);
  if (ad.rank <= 16) return launch_tile<1, 2>(P, sms, spare, stream);
  if (ad.rank <= 32) return launch_tile<1, 4>(P, sms, spare, stream);
  if (ad.rank <= 64) return launch_tile<1, 8>(P, sms, spare, stream);
  return launch_tile<1, 16>(P, sms, spare, stream);
}

cudaError_t launch_linear_small(const PackedLayer& L, const AdapterView* ad, int T, const int* row_adapter,
                                const bf16* x, long long ldx, bf16* y, long long ldy, const float* h,
                                cudaStream_t stream) {
  SmallParams P = {};
  P.L = L;
  P.x = x;
  P.ldx = ldx;
  P.y = y;
  P.ldy = ldy;
  P.T = T;
  if (ad) {
    P.up = ad->out;
    P.row_adapter = row_adapter;
    P.h = h;
    P.n_adapters = ad->n;
    P.rank = ad->rank;
  }
  if (T <= 8) return launch_small<1, 1>(P, stream);
  // more rows: tiles of 32 channels read them half as often, where the layer has enough channels for that
  return L.d_out >= 8192 ? launch_small<2, 2>(P, stream) : launch_small<1, 2>(P, stream);
}

}  // namespace admmq
