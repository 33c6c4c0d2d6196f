// The end of attention over the cache where a row's positions were shared out over several CTAs (cache_schedule.cuh).
// Bound: latency, and reading the partial results (fp32) where there are many rows.
#include "cache.h"

namespace admmq {
namespace {

constexpr float LN2 = 0.693147180559945309f;

// Adds up the partial results of a (tile, head) in the order of their CTAs.  A warp a row.
// tile_rows: rows of a tile, `per` of them to one of the plan's tiles.
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ AttendArgs a, const int4* tiles, int tile_rows, int per) {
  pdl_launch();
  pdl_wait();
  const int first = blockIdx.x, lane = threadIdx.x & 31, r = blockIdx.y * 4 + (threadIdx.x >> 5), p = a.c.p;
  const int4 join = a.joins[first];
  if (join.x < 0) return;
  int4 job = __ldg(tiles + join.x / per);
  job.y += join.x % per * tile_rows;
  const int group = a.pl.group, nr = min(tile_rows, job.w * group - job.y);
  if (r >= nr) return;
  const int last = join.z;
  // slot of CTA c: 1 where the (tile, head) begins, 0 after
  float m = -INFINITY;
  for (int c = first + lane; c <= last; c += 32) m = fmaxf(m, a.part_ml[(2 * c + (c == first)) * tile_rows + r].x);
  m = warp_max(m);
  const float ref = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  const int at = 4 * lane;
#pragma unroll 4
  for (int c = first; c <= last; ++c) {
    const long long row = (2 * c + (c == first)) * tile_rows + r;
    const float2 ml = a.part_ml[row];
    const float k = exp2_fast(ml.x - ref);
    l = fmaf(ml.y, k, l);
    const float* src = a.part + row * p + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (at + 128 * i < a.c.d) {
        const float4 x = *reinterpret_cast<const float4*>(src + 128 * i);
        acc[i].x = fmaf(x.x, k, acc[i].x);
        acc[i].y = fmaf(x.y, k, acc[i].y);
        acc[i].z = fmaf(x.z, k, acc[i].z);
        acc[i].w = fmaf(x.w, k, acc[i].w);
      }
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int pr = job.y + r, head = join.y * group + pr % group;
  const long long row = job.z + pr / group;
  bf16* dst = a.out + row * a.out_row + head * a.out_head + at;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (at + 128 * i < a.c.d)
      *reinterpret_cast<uint2*>(dst + 128 * i) =
          make_uint2(float2_to_bf16x2(acc[i].x * inv, acc[i].y * inv), float2_to_bf16x2(acc[i].z * inv, acc[i].w * inv));
  if (lane == 0 && a.lse) a.lse[row * (a.c.heads * group) + head] = l == 0.0f ? -INFINITY : m * LN2 + logf(l);
}

}  // namespace

cudaError_t launch_cache_join(const AttendArgs& a, bool many, int sms, cudaStream_t stream) {
  const int rows = many ? many_rows(a.c.p) : FEW_ROWS, per = many ? MANY_ROWS / rows : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sms * (many ? 1 : few_ctas(a.c.p)) - 1, rows / 4);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_kernel, a, many ? a.pl.big : a.pl.small, rows, per);
}

}  // namespace admmq
