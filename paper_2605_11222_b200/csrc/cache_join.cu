// The end of attention over the cache where a row's positions were shared out over several CTAs (cache_schedule.cuh):
//   out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c,  M = max_c m_c,  over the CTAs c in their order.
// Bound: latency.  Few rows are shared out over many CTAs: a block of four warps takes a row, every fourth part each with four
// loads under way, and adds up in shared memory (a warp that took the 55 parts of a request of 32768 tokens one after the
// other needed 32 us).  Many rows have few parts: a warp takes two rows at once, two parts of each under way.  Small blocks of
// few registers, so that all of them are there when the attention ends (64 ragged requests of 3000 tokens on average, the whole
// call: 76.5 us; 80 with blocks of four rows, of which an SM holds one; 32 requests with 4 new rows each: 62 and 70).
#include "cache.h"

namespace admmq {
namespace {

constexpr float LN2 = 0.693147180559945309f;

// tile_rows: rows of a tile.  H: 128-value columns of a row.  SLOTS groups of WPR warps, each with RPW rows, AT_ONCE parts of them
// at once.
template <int H, int SLOTS, int WPR, int RPW, int AT_ONCE>
__global__ void __launch_bounds__(32 * WPR * SLOTS) join_kernel(const __grid_constant__ AttendArgs a, int tile_rows) {
  static_assert(WPR == 1 || RPW == 1, "one or the other");
  __shared__ __align__(16) float sums[WPR > 1 ? SLOTS : 1][WPR][128 * H];
  __shared__ float totals[SLOTS][WPR];
  pdl_wait();
  pdl_launch();                                      // (not before: the next call's CTAs would come while the attention still
                                                     // has its places; two calls over 2 x 100001 tokens in turn 103 us each, 78 so)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = warp / WPR, w = warp % WPR;
  const int r0 = (blockIdx.y * SLOTS + slot) * RPW, p = a.c.p, d = a.c.d;
  const Join join = a.joins[blockIdx.x];
  const int first = join.first, parts = join.last - first + 1;
  if (parts == 1) return;                            // (the same for the whole block)
  const int group = a.pl.group, nr = join.rows;
  if (blockIdx.y * SLOTS * RPW >= nr) return;
  // row r of part i: slot 1 of its CTA where the (tile, head) begins, 0 after
  // (numbers of 32 bits: a few hundred CTAs' rows of at most 256 values)
  auto row_of = [&](int i, int r) { return (2 * (first + i) + (i == 0)) * tile_rows + r; };
  auto on = [&](int c) { return 4 * lane + 128 * c < d; };
  float m[RPW], l[RPW];
  float4 acc[RPW][H];
#pragma unroll
  for (int q = 0; q < RPW; ++q) {
    m[q] = -INFINITY;
    l[q] = 0.0f;
#pragma unroll
    for (int c = 0; c < H; ++c) acc[q][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (r0 < nr) {
    float4 x[AT_ONCE][RPW][H];
    float2 ml[AT_ONCE][RPW];
    auto fetch = [&](int i0) {
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e)
#pragma unroll
        for (int q = 0; q < RPW; ++q) {
          const int i = i0 + e * WPR;
          const int row = row_of(i, min(r0 + q, nr - 1));
          ml[e][q] = i < parts ? a.part_ml[row] : make_float2(-INFINITY, 0.0f);
          const float* src = a.part + (unsigned)(row * p + 4 * lane);
#pragma unroll
          for (int c = 0; c < H; ++c)
            x[e][q][c] = on(c) && i < parts ? *reinterpret_cast<const float4*>(src + 128 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    float top[RPW];
#pragma unroll
    for (int q = 0; q < RPW; ++q) top[q] = lane < parts ? a.part_ml[row_of(lane, min(r0 + q, nr - 1))].x : -INFINITY;
    fetch(w);                                        // (under way with the maxima)
    for (int i = lane + 32; i < parts; i += 32)
#pragma unroll
      for (int q = 0; q < RPW; ++q) top[q] = fmaxf(top[q], a.part_ml[row_of(i, min(r0 + q, nr - 1))].x);
#pragma unroll
    for (int q = 0; q < RPW; ++q) m[q] = warp_max(top[q]);
    for (int i0 = w; i0 < parts; i0 += WPR * AT_ONCE) {
      if (i0 > w) fetch(i0);
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e)
#pragma unroll
        for (int q = 0; q < RPW; ++q) {
          const float k = exp2_fast(ml[e][q].x - (m[q] == -INFINITY ? 0.0f : m[q]));
          l[q] = fmaf(ml[e][q].y, k, l[q]);
#pragma unroll
          for (int c = 0; c < H; ++c) {
            acc[q][c].x = fmaf(x[e][q][c].x, k, acc[q][c].x);
            acc[q][c].y = fmaf(x[e][q][c].y, k, acc[q][c].y);
            acc[q][c].z = fmaf(x[e][q][c].z, k, acc[q][c].z);
            acc[q][c].w = fmaf(x[e][q][c].w, k, acc[q][c].w);
          }
        }
    }
  }
  if (WPR > 1) {
#pragma unroll
    for (int c = 0; c < H; ++c) *reinterpret_cast<float4*>(&sums[slot][w][4 * lane + 128 * c]) = acc[0][c];
    if (lane == 0) totals[slot][w] = l[0];
    __syncthreads();
    if (w > 0) return;
    l[0] = 0.0f;
#pragma unroll
    for (int v = 0; v < WPR; ++v) l[0] += totals[slot][v];
#pragma unroll
    for (int c = 0; c < H; ++c) {
      acc[0][c] = *reinterpret_cast<const float4*>(&sums[slot][0][4 * lane + 128 * c]);
#pragma unroll
      for (int v = 1; v < WPR; ++v) {
        const float4 x = *reinterpret_cast<const float4*>(&sums[slot][v][4 * lane + 128 * c]);
        acc[0][c].x += x.x;
        acc[0][c].y += x.y;
        acc[0][c].z += x.z;
        acc[0][c].w += x.w;
      }
    }
  }
#pragma unroll
  for (int q = 0; q < RPW; ++q) {
    if (r0 + q >= nr) return;
    const float inv = l[q] == 0.0f ? 0.0f : 1.0f / l[q];
    const int pr = join.row0 + r0 + q, head = join.head * group + pr % group;
    const long long row = join.first_row + pr / group;
    bf16* dst = a.out + row * a.out_row + head * a.out_head + 4 * lane;
#pragma unroll
    for (int c = 0; c < H; ++c)
      if (on(c))
        *reinterpret_cast<uint2*>(dst + 128 * c) = make_uint2(float2_to_bf16x2(acc[q][c].x * inv, acc[q][c].y * inv),
                                                              float2_to_bf16x2(acc[q][c].z * inv, acc[q][c].w * inv));
    if (lane == 0 && a.lse) a.lse[row * (a.c.heads * group) + head] = l[q] == 0.0f ? -INFINITY : m[q] * LN2 + logf(l[q]);
  }
}

template <int H, int SLOTS, int WPR, int RPW, int AT_ONCE>
cudaError_t launch(const AttendArgs& a, int joins, int rows, int max_rows, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(joins, (max_rows + SLOTS * RPW - 1) / (SLOTS * RPW));
  cfg.blockDim = dim3(32 * WPR * SLOTS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_kernel<H, SLOTS, WPR, RPW, AT_ONCE>, a, rows);
}
template <int H>
cudaError_t launch(const AttendArgs& a, bool many, int joins, cudaStream_t stream) {
  return many ? launch<H, 4, 1, 2, 2>(a, joins, many_rows(a.c.p), many_rows(a.c.p), stream)
              : launch<H, 1, 4, 1, 4>(a, joins, FEW_ROWS, a.pl.small_rows, stream);
}

}  // namespace

cudaError_t launch_cache_join(const AttendArgs& a, bool many, int sms, cudaStream_t stream) {
  const int joins = a.by_piece ? pieces_of(a, many) : attend_ctas(a.c.p, many, sms);
  return a.c.p <= 128 ? launch<1>(a, many, joins, stream) : launch<2>(a, many, joins, stream);
}

}  // namespace admmq
