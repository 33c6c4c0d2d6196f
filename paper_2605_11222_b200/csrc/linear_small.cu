// The projection for a few rows (decoding), and the contraction of the rows with their adapters.
//
// linear_small: y[t][j] = sum_i x[t][i] W[j][i], up to 16 rows.  Bound: memory, half a byte a weight.  With
// W = z0 + Delta k a group of input channels contributes  Delta sum k x + z0 sum x, so the tensor cores multiply the
// codes themselves: 0x4300 | k is the bf16 number 128 + k, two codes leave a packed word per shift and mask, and
//   y = sum over groups of  Delta (sum (128 + k) x) + (z0 - 128 Delta) sum x
// in fp32, without a rounding of any weight.  sum x comes from a second product with a tile of ones.  (The offset
// 128 costs 7 of the 24 bits of the fp32 sums: 2^-17 relative, under the 2^-9 of the output.)
// A CTA of 8 warps owns 16 output channels for up to 8 rows, 32 for more (then the rows are read from L2 half as
// often); the warps split the input channels, a warp's loads of UNROLL blocks of codes leave together, and the sums
// meet in shared memory.  Channels are taken in an order that lets a thread read 16 of them from consecutive
// addresses for the codes and for x alike: a product over them does not ask for their order.
//
// shrink: h[t][r] = scale_a sum_i x[t][i] in_a[r][i].  Bound: memory, one pass over the rows and over the adapters in
// use.  Two forms: a CTA for each row and 8 ranks (a warp a rank) for few rows, and tiles of 16 or 32 rows on mma.sync
// for more, where the passes over a tile are one per distinct adapter in it.
#include <cooperative_groups.h>

#include "adapt.h"

namespace cg = cooperative_groups;

namespace admmq {
namespace {

constexpr int THREADS = 256, WARPS = 8;

// ------------------------------------------------------------------ few rows: the projection
struct SmallParams {
  PackedLayer L;
  const bf16* x;
  long long ldx;
  bf16* y;
  long long ldy;
  int T;
  const bf16* up;                 // adapters' output side [n][rank][d_out], NULL: none
  const int* row_adapter;
  const float* h;                 // [T][rank]
  int n_adapters, rank;
};

// MT tiles of 16 channels, NT tiles of 8 rows.
template <int MT, int NT>
__global__ void __launch_bounds__(THREADS) linear_small_kernel(const __grid_constant__ SmallParams P) {
  constexpr int UNROLL = 4;
  __shared__ float red[WARPS][NT * 8][MT * 16 + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, q = lane & 3;
  const int j0 = blockIdx.x * 16 * MT;
  const int p = P.L.d_out, n = P.L.d_in;
  const int ib0 = P.L.nib * warp / WARPS, ib1 = P.L.nib * (warp + 1) / WARPS;

  int row[MT][2];                                  // output channels of this thread, kept inside the matrix
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    row[m][0] = min(j0 + 16 * m + g, p - 1);
    row[m][1] = min(j0 + 16 * m + g + 8, p - 1);
  }
  float y[MT][NT][4], acc[MT][NT][4], sx[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sx[t][e] = 0.0f;
#pragma unroll
      for (int m = 0; m < MT; ++m) y[m][t][e] = acc[m][t][e] = 0.0f;
    }
  const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

  for (int ib = ib0; ib < ib1; ib += UNROLL) {
    uint2 code[UNROLL][MT][2];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          if (ib + u < ib1)
            code[u][m][hh] = __ldg(reinterpret_cast<const uint2*>(
                                       P.L.codes + ((long long)(ib + u) * p + row[m][hh]) * BLOCK_WORDS) + q);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (ib + u >= ib1) break;
      const int i = (ib + u) * CODE_BLOCK + 16 * q;
      uint4 xv[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bf16* px = P.x + (long long)(8 * t + g) * P.ldx + i;
        const bool in = 8 * t + g < P.T;
        xv[t][0] = in && i < n ? __ldg(reinterpret_cast<const uint4*>(px)) : make_uint4(0, 0, 0, 0);
        xv[t][1] = in && i + 8 < n ? __ldg(reinterpret_cast<const uint4*>(px) + 1) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int s = 0; s < 2; ++s) {              // 16 channels: pairs 2 s and 2 s + 1 of the word
          uint32_t b[NT][2];
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            b[t][0] = s == 0 ? xv[t][w].x : xv[t][w].z;
            b[t][1] = s == 0 ? xv[t][w].y : xv[t][w].w;
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const uint32_t c0 = w == 0 ? code[u][m][0].x : code[u][m][0].y;
            const uint32_t c1 = w == 0 ? code[u][m][1].x : code[u][m][1].y;
            const uint32_t a[4] = {((c0 >> (8 * s)) & 0x000F000Fu) | 0x43004300u,
                                   ((c1 >> (8 * s)) & 0x000F000Fu) | 0x43004300u,
                                   ((c0 >> (8 * s + 4)) & 0x000F000Fu) | 0x43004300u,
                                   ((c1 >> (8 * s + 4)) & 0x000F000Fu) | 0x43004300u};
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_bf16(acc[m][t], a, b[t][0], b[t][1]);
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_bf16(sx[t], ones, b[t][0], b[t][1]);
        }
      // the end of a group (or of this warp's share): fold its sums into y
      const int grp = (ib + u) * CODE_BLOCK / P.L.gs;
      if (ib + u + 1 == ib1 || (ib + u + 1) * CODE_BLOCK / P.L.gs != grp) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float2 g0 = __ldg(P.L.grid + (long long)grp * p + row[m][0]);
          const float2 g1 = __ldg(P.L.grid + (long long)grp * p + row[m][1]);
          const float z0 = fmaf(-128.0f, g0.x, g0.y), z1 = fmaf(-128.0f, g1.x, g1.y);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            y[m][t][0] += fmaf(g0.x, acc[m][t][0], z0 * sx[t][0]);
            y[m][t][1] += fmaf(g0.x, acc[m][t][1], z0 * sx[t][1]);
            y[m][t][2] += fmaf(g1.x, acc[m][t][2], z1 * sx[t][2]);
            y[m][t][3] += fmaf(g1.x, acc[m][t][3], z1 * sx[t][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][t][e] = 0.0f;
          }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sx[t][e] = 0.0f;
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      red[warp][8 * t + 2 * q][16 * m + g] = y[m][t][0];
      red[warp][8 * t + 2 * q + 1][16 * m + g] = y[m][t][1];
      red[warp][8 * t + 2 * q][16 * m + g + 8] = y[m][t][2];
      red[warp][8 * t + 2 * q + 1][16 * m + g + 8] = y[m][t][3];
    }
  __syncthreads();
  if (P.up != nullptr) pdl_wait();                 // h is complete from here on
  for (int o = threadIdx.x; o < P.T * 16 * MT; o += THREADS) {
    const int t = o / (16 * MT), m = o % (16 * MT), j = j0 + m;
    if (j >= p) continue;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) v += red[w][t][m];
    if (P.up != nullptr) {
      const int a = row_adapter_of(P.row_adapter, t, P.n_adapters);
      if (a >= 0) {
        const bf16* up = P.up + (long long)a * P.rank * p + j;
        const float* h = P.h + (long long)t * P.rank;
        float d = 0.0f;
#pragma unroll 8
        for (int r = 0; r < P.rank; ++r) d = fmaf(h[r], __bfloat162float(up[(long long)r * p]), d);
        v += d;
      }
    }
    P.y[(long long)t * P.ldy + j] = __float2bfloat16_rn(v);
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

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float s) {
  const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 x = bf16x2_to_float2(av[e]), y = bf16x2_to_float2(bv[e]);
    s = fmaf(x.x, y.x, fmaf(x.y, y.y, s));
  }
  return s;
}

// One row and 8 ranks a CTA, a warp a rank.
__global__ void __launch_bounds__(THREADS) shrink_rows_kernel(const __grid_constant__ ShrinkParams P) {
  pdl_launch();
  const long long t = blockIdx.x;
  const int r = blockIdx.y * WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int a = row_adapter_of(P.row_adapter, t, P.n);
  float v = 0.0f;
  if (a >= 0) {
    const bf16* x = P.x + t * P.ldx;
    const bf16* m = P.mat + ((long long)a * P.rank + r) * P.K;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = lane * 8; i < P.K; i += 4 * 256) {
      uint4 xv[4], mv[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool in = i + 256 * u < P.K;
        xv[u] = in ? __ldg(reinterpret_cast<const uint4*>(x + i + 256 * u)) : make_uint4(0, 0, 0, 0);
        mv[u] = in ? __ldg(reinterpret_cast<const uint4*>(m + i + 256 * u)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] = dot8(xv[u], mv[u], s[u]);
    }
    v = warp_sum((s[0] + s[1]) + (s[2] + s[3])) * P.scale[a];
  }
  if (lane == 0) P.h[t * P.rank + r] = v;
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
    const int stride = WARPS * 32 * shares;
    for (int k0 = (share * WARPS + warp) * 32; k0 < P.K; k0 += UNR * stride) {
      uint4 av[UNR][MT][2], bv[UNR][NT];
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        const int i = k0 + u * stride + 8 * q;
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
cudaError_t launch_tile(const ShrinkParams& P, int sms, cudaStream_t stream) {
  constexpr int BYTES = (WARPS + 1) * 16 * MT * 8 * NT * 4;
  const cudaError_t e = ensure_dynamic_smem((const void*)shrink_tile_kernel<MT, NT>, BYTES);
  if (e != cudaSuccess) return e;
  const long long tiles = (P.T + 16 * MT - 1) / (16 * MT);
  // CTAs of a tile: as many as bring two to every multiprocessor and leave each at least two steps of all its warps
  int shares = 1;
  while (shares < 8 && tiles * shares < 2 * sms && P.K >= 2 * WARPS * 32 * 2 * shares) shares *= 2;
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
cudaError_t launch_small(const SmallParams& P, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((P.L.d_out + 16 * MT - 1) / (16 * MT));
  cfg.blockDim = dim3(THREADS);
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
                          const int* row_adapter, float* h, cudaStream_t stream) {
  const ShrinkParams P = {x, ldx, T, K, ad.in, ad.scale, ad.n, ad.rank, row_adapter, h};
  if (T <= SHRINK_ROWS_MAX) {
    shrink_rows_kernel<<<dim3((unsigned)T, ad.rank / 8), THREADS, 0, stream>>>(P);
    return cudaGetLastError();
  }
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  // Tiles of 32 rows read the adapters half as often; tiles of 16 meet fewer distinct adapters and are more.
  if (T > 1024) {
    if (ad.rank <= 8) return launch_tile<2, 1>(P, sms, stream);
    if (ad.rank <= 16) return launch_tile<2, 2>(P, sms, stream);
    if (ad.rank <= 32) return launch_tile<2, 4>(P, sms, stream);
    if (ad.rank <= 64) return launch_tile<2, 8>(P, sms, stream);
  }
  if (ad.rank <= 8) return launch_tile<1, 1>(P, sms, stream);
  if (ad.rank <= 16) return launch_tile<1, 2>(P, sms, stream);
  if (ad.rank <= 32) return launch_tile<1, 4>(P, sms, stream);
  if (ad.rank <= 64) return launch_tile<1, 8>(P, sms, stream);
  return launch_tile<1, 16>(P, sms, stream);
}

cudaError_t launch_linear_small(const PackedLayer& L, const AdapterView* ad, int T, const int* row_adapter,
                                const bf16* x, long long ldx, bf16* y, long long ldy, const float* h,
                                cudaStream_t stream) {
  const SmallParams P = {L, x, ldx, y, ldy, T, ad ? ad->out : nullptr, row_adapter, h, ad ? ad->n : 0, ad ? ad->rank : 0};
  if (T <= 8) return launch_small<1, 1>(P, stream);
  return launch_small<2, 2>(P, stream);
}

}  // namespace admmq
