// The end of attention over the cache where a row's positions were shared out over several CTAs (cache_schedule.cuh):
//   out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c,  M = max_c m_c,  over the CTAs c in their order.
// Bound: latency.  WPR warps take a row, every WPR-th part each with eight loads under way, and add up in shared memory (a
// warp that took its 55 parts of one request of 32768 tokens one after the other needed 32 us).
#include "cache.h"

namespace admmq {
namespace {

constexpr float LN2 = 0.693147180559945309f;
constexpr int ROWS_AT_ONCE = 4;

// tile_rows: rows of a tile, `per` of them to one of the plan's tiles.
template <int WPR>
__global__ void __launch_bounds__(32 * WPR * ROWS_AT_ONCE) join_kernel(const __grid_constant__ AttendArgs a, const int4* tiles, int tile_rows, int per) {
  __shared__ __align__(16) float sums[WPR > 1 ? ROWS_AT_ONCE : 1][WPR][256];
  __shared__ float totals[ROWS_AT_ONCE][WPR];
  pdl_launch();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = warp / WPR, w = warp % WPR;
  const int r = blockIdx.y * ROWS_AT_ONCE + slot, p = a.c.p, d = a.c.d;
  const int4 join = a.joins[blockIdx.x];
  const int first = join.z, parts = join.w - first + 1;
  if (parts == 1) return;                            // (the same for the whole block)
  int4 job = __ldg(tiles + join.x / per);
  job.y += join.x % per * tile_rows;
  const int group = a.pl.group, nr = min(tile_rows, job.w * group - job.y);
  if (blockIdx.y * ROWS_AT_ONCE >= nr) return;
  // row of part i: slot 1 of its CTA where the (tile, head) begins, 0 after
  auto row_of = [&](int i) { return (long long)(2 * (first + i) + (i == 0)) * tile_rows + r; };
  float m = -INFINITY, l = 0.0f;
  float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  if (r < nr) {
    for (int i = lane; i < parts; i += 32) m = fmaxf(m, a.part_ml[row_of(i)].x);
    m = warp_max(m);
    const float ref = m == -INFINITY ? 0.0f : m;
    const bool on[2] = {4 * lane < d, 4 * lane + 128 < d};
    constexpr int AT_ONCE = 8;
    for (int i0 = w; i0 < parts; i0 += WPR * AT_ONCE) {
      float4 x[AT_ONCE][2];
      float2 ml[AT_ONCE];
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        const int i = i0 + e * WPR;
        const long long row = row_of(min(i, parts - 1));
        ml[e] = a.part_ml[row];
        if (i >= parts) ml[e] = make_float2(-INFINITY, 0.0f);
        const float* src = a.part + row * p + 4 * lane;
#pragma unroll
        for (int k = 0; k < 2; ++k) x[e][k] = on[k] && i < parts ? *reinterpret_cast<const float4*>(src + 128 * k) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        const float k = exp2_fast(ml[e].x - ref);
        l = fmaf(ml[e].y, k, l);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          acc[c].x = fmaf(x[e][c].x, k, acc[c].x);
          acc[c].y = fmaf(x[e][c].y, k, acc[c].y);
          acc[c].z = fmaf(x[e][c].z, k, acc[c].z);
          acc[c].w = fmaf(x[e][c].w, k, acc[c].w);
        }
      }
    }
  }
  if (WPR > 1) {
#pragma unroll
    for (int c = 0; c < 2; ++c) *reinterpret_cast<float4*>(&sums[slot][w][4 * lane + 128 * c]) = acc[c];
    if (lane == 0) totals[slot][w] = l;
    __syncthreads();
    if (w > 0 || r >= nr) return;
    l = 0.0f;
#pragma unroll
    for (int v = 0; v < WPR; ++v) l += totals[slot][v];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      acc[c] = *reinterpret_cast<const float4*>(&sums[slot][0][4 * lane + 128 * c]);
#pragma unroll
      for (int v = 1; v < WPR; ++v) {
        const float4 x = *reinterpret_cast<const float4*>(&sums[slot][v][4 * lane + 128 * c]);
        acc[c].x += x.x;
        acc[c].y += x.y;
        acc[c].z += x.z;
        acc[c].w += x.w;
      }
    }
  } else if (r >= nr) {
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int pr = job.y + r, head = join.y * group + pr % group;
  const long long row = job.z + pr / group;
  bf16* dst = a.out + row * a.out_row + head * a.out_head + 4 * lane;
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (4 * lane + 128 * c < d)
      *reinterpret_cast<uint2*>(dst + 128 * c) =
          make_uint2(float2_to_bf16x2(acc[c].x * inv, acc[c].y * inv), float2_to_bf16x2(acc[c].z * inv, acc[c].w * inv));
  if (lane == 0 && a.lse) a.lse[row * (a.c.heads * group) + head] = l == 0.0f ? -INFINITY : m * LN2 + logf(l);
}

template <int WPR>
cudaError_t launch(const AttendArgs& a, int joins, const int4* tiles, int rows, int per, int max_rows, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(joins, (max_rows + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE);
  cfg.blockDim = dim3(32 * WPR * ROWS_AT_ONCE);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_kernel<WPR>, a, tiles, rows, per);
}

}  // namespace

cudaError_t launch_cache_join(const AttendArgs& a, bool many, int sms, cudaStream_t stream) {
  const int rows = many ? many_rows(a.c.p) : FEW_ROWS;
  const int joins = a.by_piece ? pieces_of(a, many) : attend_ctas(a.c.p, many, sms);
  return many ? launch<1>(a, joins, a.pl.big, rows, MANY_ROWS / rows, rows, stream)
              : launch<4>(a, joins, a.pl.small, rows, 1, a.pl.small_rows, stream);
}

}  // namespace admmq
