// Activation checkpoints in 8 bits: for every row and block of 128 channels  scale = max |x| / 127,
// code = rint(x / scale);  x^ = scale * code.
//
// Bound: memory, 3 bytes a bf16 value (2 read, 1 written) and 4 bytes a block.  Sixteen threads hold one block, 8
// channels each, so that the maximum is four shuffles away and nothing is read twice; a thread takes UNROLL blocks at
// once, which keeps 64 (bf16) or 128 (fp32) bytes a thread in flight.
#include "adapt.h"

namespace admmq {
namespace {

constexpr int BLOCK = ADMMQ_CHECKPOINT_BLOCK;
constexpr int LANES = BLOCK / 8;            // threads of one block
constexpr int THREADS = 256;
constexpr int UNROLL = 4;
constexpr int PAIRS = THREADS / LANES * UNROLL;   // (row, block) pairs of one CTA

struct Place {
  long long row;
  int blk;
};
// Pair `off` after the CTA's first one; nb blocks a row.
__device__ __forceinline__ Place place_of(long long row0, unsigned blk0, unsigned off, unsigned nb) {
  const unsigned s = blk0 + off, r = s / nb;
  return {row0 + r, (int)(s - r * nb)};
}

template <bool BF16>
__global__ void __launch_bounds__(THREADS)
checkpoint_save_kernel(const void* __restrict__ x, long long T, int width, long long ldx, int nb,
                       int8_t* __restrict__ codes, float* __restrict__ scale) {
  const long long first = (long long)blockIdx.x * PAIRS;
  const long long row0 = first / nb;
  const unsigned blk0 = (unsigned)(first - row0 * nb);
  const int sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  uint4 raw[UNROLL][BF16 ? 1 : 2];
  Place at[UNROLL];
  bool on[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    at[u] = place_of(row0, blk0, (unsigned)(u * (THREADS / LANES) + sub), (unsigned)nb);
    const int i = at[u].blk * BLOCK + lane * 8;
    on[u] = at[u].row < T && i < width;       // width is a multiple of 8: all eight channels or none
    const char* p = (const char*)x + (at[u].row * ldx + i) * (BF16 ? 2 : 4);
#pragma unroll
    for (int q = 0; q < (BF16 ? 1 : 2); ++q) raw[u][q] = on[u] ? ldg_stream(p + 16 * q) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    float v[8];
    if (BF16) {
      const uint32_t w[4] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = bf16x2_to_float2(w[e]);
        v[2 * e] = f.x;
        v[2 * e + 1] = f.y;
      }
    } else {
      const uint4* r = raw[u];
      const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[BF16 ? 0 : 1].x, r[BF16 ? 0 : 1].y, r[BF16 ? 0 : 1].z,
                             r[BF16 ? 0 : 1].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(w[e]);
    }
    // The order of the magnitudes' bit patterns is that of the magnitudes, with infinity and NaN on top: an integer
    // maximum finds the largest value and does not lose a NaN.
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool finite = top < 0x7f800000u;
    const float s = finite ? __fdiv_rn(__uint_as_float(top), 127.0f) : __int_as_float(0x7fc00000);
    if (!on[u]) continue;
    uint32_t out[2] = {0u, 0u};
    if (finite && s > 0.0f) {
      // The quotient as the division rounds it: codes do not depend on how a reciprocal is formed.  (A maximum so
      // small that the scale is subnormal leaves quotients above 127: the clamp.)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = min(127, max(-127, __float2int_rn(__fdiv_rn(v[e], s))));
        out[e >> 2] |= (uint32_t)(k & 0xff) << (8 * (e & 3));
      }
    }
    *reinterpret_cast<uint2*>(codes + at[u].row * width + at[u].blk * BLOCK + lane * 8) = make_uint2(out[0], out[1]);
    if (lane == 0) scale[at[u].row * nb + at[u].blk] = s;
  }
}

template <bool BF16>
__global__ void __launch_bounds__(THREADS)
checkpoint_restore_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scale, long long T, int width,
                          int nb, void* __restrict__ out, long long ldo) {
  const long long first = (long long)blockIdx.x * PAIRS;
  const long long row0 = first / nb;
  const unsigned blk0 = (unsigned)(first - row0 * nb);
  const int sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  uint2 raw[UNROLL];
  float s[UNROLL];
  Place at[UNROLL];
  bool on[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    at[u] = place_of(row0, blk0, (unsigned)(u * (THREADS / LANES) + sub), (unsigned)nb);
    const int i = at[u].blk * BLOCK + lane * 8;
    on[u] = at[u].row < T && i < width;
    raw[u] = on[u] ? __ldg(reinterpret_cast<const uint2*>(codes + at[u].row * width + i)) : make_uint2(0, 0);
    s[u] = on[u] ? __ldg(scale + at[u].row * nb + at[u].blk) : 0.0f;
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (!on[u]) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = e < 4 ? raw[u].x : raw[u].y;
      v[e] = s[u] * (float)(int8_t)(w >> (8 * (e & 3)));
    }
    char* p = (char*)out + (at[u].row * ldo + at[u].blk * BLOCK + lane * 8) * (BF16 ? 2 : 4);
    if (BF16) {
      uint4 o;
      o.x = float2_to_bf16x2(v[0], v[1]);
      o.y = float2_to_bf16x2(v[2], v[3]);
      o.z = float2_to_bf16x2(v[4], v[5]);
      o.w = float2_to_bf16x2(v[6], v[7]);
      *reinterpret_cast<uint4*>(p) = o;
    } else {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(p + 16) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
}

}  // namespace

cudaError_t launch_checkpoint_save(const void* x, int is_bf16, long long T, int width, long long ldx, int8_t* codes,
                                   float* scale, cudaStream_t stream) {
  const int nb = (width + BLOCK - 1) / BLOCK;
  const long long ctas = (T * nb + PAIRS - 1) / PAIRS;
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (is_bf16)
    checkpoint_save_kernel<true><<<(unsigned)ctas, THREADS, 0, stream>>>(x, T, width, ldx, nb, codes, scale);
  else
    checkpoint_save_kernel<false><<<(unsigned)ctas, THREADS, 0, stream>>>(x, T, width, ldx, nb, codes, scale);
  return cudaGetLastError();
}

cudaError_t launch_checkpoint_restore(const int8_t* codes, const float* scale, long long T, int width, void* out,
                                      int is_bf16, long long ldo, cudaStream_t stream) {
  const int nb = (width + BLOCK - 1) / BLOCK;
  const long long ctas = (T * nb + PAIRS - 1) / PAIRS;
  if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (is_bf16)
    checkpoint_restore_kernel<true><<<(unsigned)ctas, THREADS, 0, stream>>>(codes, scale, T, width, nb, out, ldo);
  else
    checkpoint_restore_kernel<false><<<(unsigned)ctas, THREADS, 0, stream>>>(codes, scale, T, width, nb, out, ldo);
  return cudaGetLastError();
}

}  // namespace admmq
