// Activation checkpoints in 8 bits: for every row and block of 128 channels  scale = max |x| / 127,
// code = rint(x / scale);  x^ = scale * code.
//
// Bound: memory, 3 bytes a bf16 value (2 read, 1 written) and 4 bytes a block.  A block is held by eight threads (to save)
// or sixteen (to restore), 8 channels at a time, so that the maximum is a few shuffles away and nothing is read twice; a
// thread's loads all leave together, 64 (bf16) or 128 (fp32) bytes to save.  At three bytes a value the instructions count
// (a first form with eight divisions a thread and scalar arithmetic issued 170 for every 8 values and ran at 45 % of the
// copy rate): maxima and products run on packed pairs, and a scale's division and reciprocal are made by half the
// threads, one of two blocks each.
#include "adapt.h"

namespace admmq {
namespace {

constexpr int BLOCK = ADMMQ_CHECKPOINT_BLOCK;
constexpr int LANES = BLOCK / 8;            // threads of one block
constexpr int THREADS = 256;
constexpr int UNROLL = 4;
constexpr int PAIRS = THREADS / LANES * UNROLL;   // (row, block) pairs of one CTA

// The (row, block) pairs of a CTA: consecutive ones, nb to a row.
struct Pairs {
  long long row0;
  uint32_t blk0, nb, inv;                   // inv = ceil(2^32 / nb): exact quotients for numbers below 2^32 / nb
  __device__ __forceinline__ Pairs(uint32_t nb_, uint32_t inv_) : nb(nb_), inv(inv_) {
    const uint32_t first = blockIdx.x * (uint32_t)PAIRS, r = first / nb;      // (at most 2^31 pairs)
    row0 = r;
    blk0 = first - r * nb;
  }
  __device__ __forceinline__ void at(uint32_t off, long long& row, int& blk) const {
    const uint32_t n = blk0 + off, r = nb == 1 ? n : __umulhi(n, inv);
    row = row0 + r;
    blk = (int)(n - r * nb);
  }
};

// The largest magnitude's bit pattern of this thread's 8 values.  (The order of the patterns is that of the
// magnitudes, with infinity and NaN on top: an integer maximum finds the largest value and does not lose a NaN.)
// bf16: as the upper 16 bits of an fp32 number.
template <bool BF16>
__device__ __forceinline__ uint32_t top8(const uint4* r) {
  if (BF16) {
    uint32_t t = __vmaxu2(__vmaxu2(r->x & 0x7fff7fffu, r->y & 0x7fff7fffu), __vmaxu2(r->z & 0x7fff7fffu, r->w & 0x7fff7fffu));
    return max(t & 0xffffu, t >> 16);
  }
  uint32_t t = 0;
#pragma unroll
  for (int q = 0; q < 2; ++q)
    t = max(t, max(max(r[q].x & 0x7fffffffu, r[q].y & 0x7fffffffu), max(r[q].z & 0x7fffffffu, r[q].w & 0x7fffffffu)));
  return t;
}

// A block's eight threads hold channels 8 lane .. + 7 of its two halves each.
template <bool BF16>
__global__ void __launch_bounds__(THREADS)
checkpoint_save_kernel(const void* __restrict__ x, long long T, int width, long long ldx, uint32_t nb, uint32_t nb_inv,
                       int8_t* __restrict__ codes, float* __restrict__ scale) {
  constexpr int Q = BF16 ? 1 : 2;           // 16-byte loads of 8 values
  constexpr int LN = LANES / 2, TAKE = 2;   // threads of a block, blocks of a thread
  static_assert(THREADS / LN * TAKE == PAIRS, "the CTA's pairs");
  const Pairs pairs(nb, nb_inv);
  const int sub = threadIdx.x / LN, lane = threadIdx.x % LN;
  uint4 raw[TAKE][2][Q];
  long long row[TAKE];
  int blk[TAKE];
  bool on[TAKE][2];
#pragma unroll
  for (int u = 0; u < TAKE; ++u) {
    pairs.at((uint32_t)(u * (THREADS / LN) + sub), row[u], blk[u]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = blk[u] * BLOCK + h * (BLOCK / 2) + lane * 8;
      on[u][h] = row[u] < T && i < width;   // width is a multiple of 8: all eight channels or none
      const char* p = (const char*)x + (row[u] * ldx + i) * (BF16 ? 2 : 4);
#pragma unroll
      for (int q = 0; q < Q; ++q) raw[u][h][q] = on[u][h] ? ldg_stream(p + 16 * q) : make_uint4(0, 0, 0, 0);
    }
  }
  // largest magnitude of every block, in all its threads
  uint32_t top[TAKE];
#pragma unroll
  for (int u = 0; u < TAKE; ++u) top[u] = max(top8<BF16>(raw[u][0]), top8<BF16>(raw[u][1]));
  if (BF16) {                               // two blocks to a register
    uint32_t t = top[0] | top[1] << 16;
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) t = __vmaxu2(t, __shfl_xor_sync(0xffffffffu, t, o));
    top[0] = t << 16;
    top[1] = t & 0xffff0000u;
  } else {
#pragma unroll
    for (int u = 0; u < TAKE; ++u)
#pragma unroll
      for (int o = LN / 2; o > 0; o >>= 1) top[u] = max(top[u], __shfl_xor_sync(0xffffffffu, top[u], o));
  }
  // scale and reciprocal of block u: made by the threads with lane % 2 == u
  const uint32_t mine = (lane & 1) ? top[1] : top[0];
  const float my_s = mine < 0x7f800000u ? __fdiv_rn(__uint_as_float(mine), 127.0f) : __int_as_float(0x7fc00000);
  const float my_y = __frcp_rn(my_s);
#pragma unroll
  for (int u = 0; u < TAKE; ++u) {
    const float s = __shfl_sync(0xffffffffu, my_s, u, LN), y = __shfl_sync(0xffffffffu, my_y, u, LN);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!on[u][h]) continue;
      float2 v[4];
      if (BF16) {
        v[0] = bf16x2_to_float2(raw[u][h][0].x);
        v[1] = bf16x2_to_float2(raw[u][h][0].y);
        v[2] = bf16x2_to_float2(raw[u][h][0].z);
        v[3] = bf16x2_to_float2(raw[u][h][0].w);
      } else {
        const uint4 a = raw[u][h][0], b = raw[u][h][Q - 1];
        v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
        v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
        v[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
        v[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
      }
      uint32_t k[8];
      if (s > 1e-28f) {
        // code = rint(x / s) with the quotient as a division rounds it, without eight divisions: with y = RN(1 / s),
        // q0 = RN(x y) and the exact remainder e = x - q0 s, RN(q0 + e y) is the rounded quotient (Markstein 1990,
        // "Computation of elementary functions on the IBM RISC System/6000 processor").  Adding 1.5 * 2^23 rounds to a
        // whole number, ties to even, and leaves it in the low bits.
        const float2 y2 = make_float2(y, y), s2 = make_float2(-s, -s), magic = make_float2(12582912.0f, 12582912.0f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 q0 = __fmul2_rn(v[e], y2);
          const float2 t = __fadd2_rn(__ffma2_rn(__ffma2_rn(q0, s2, v[e]), y2, q0), magic);
          k[2 * e] = __float_as_uint(t.x);
          k[2 * e + 1] = __float_as_uint(t.y);
        }
      } else if (s > 0.0f) {
        // a scale so small that a remainder could underflow; one that is subnormal leaves quotients above 127: the clamp
#pragma unroll
        for (int e = 0; e < 8; ++e)
          k[e] = (uint32_t)min(127, max(-127, __float2int_rn(__fdiv_rn((e & 1) ? v[e >> 1].y : v[e >> 1].x, s))));
      } else {                              // zeros, or a scale of NaN
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = 0u;
      }
      uint2 out;
      out.x = __byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410);
      out.y = __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(codes + row[u] * width + blk[u] * BLOCK + h * (BLOCK / 2) + lane * 8) = out;
    }
    if (lane == 0 && on[u][0]) scale[row[u] * nb + blk[u]] = s;
  }
}

template <bool BF16>
__global__ void __launch_bounds__(THREADS)
checkpoint_restore_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scale, long long T, int width,
                          uint32_t nb, uint32_t nb_inv, void* __restrict__ out, long long ldo) {
  const Pairs pairs(nb, nb_inv);
  const int sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  uint2 raw[UNROLL];
  float s[UNROLL];
  long long row[UNROLL];
  int blk[UNROLL];
  bool on[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    pairs.at((uint32_t)(u * (THREADS / LANES) + sub), row[u], blk[u]);
    const int i = blk[u] * BLOCK + lane * 8;
    on[u] = row[u] < T && i < width;
    raw[u] = on[u] ? __ldg(reinterpret_cast<const uint2*>(codes + row[u] * width + i)) : make_uint2(0, 0);
    s[u] = on[u] ? __ldg(scale + row[u] * nb + blk[u]) : 0.0f;
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
    char* p = (char*)out + (row[u] * ldo + blk[u] * BLOCK + lane * 8) * (BF16 ? 2 : 4);
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

// CTAs for T rows of nb blocks (at most CHECKPOINT_MAX_BLOCKS in all), and ceil(2^32 / nb).
static unsigned plan_pairs(long long T, int nb, uint32_t* inv) {
  *inv = (uint32_t)(((1ULL << 32) + nb - 1) / nb);            // (nb = 1 does not use it)
  return (unsigned)((T * nb + PAIRS - 1) / PAIRS);
}

cudaError_t launch_checkpoint_save(const void* x, int is_bf16, long long T, int width, long long ldx, int8_t* codes,
                                   float* scale, cudaStream_t stream) {
  const int nb = (width + BLOCK - 1) / BLOCK;
  uint32_t inv;
  const unsigned ctas = plan_pairs(T, nb, &inv);
  if (is_bf16)
    checkpoint_save_kernel<true><<<ctas, THREADS, 0, stream>>>(x, T, width, ldx, nb, inv, codes, scale);
  else
    checkpoint_save_kernel<false><<<ctas, THREADS, 0, stream>>>(x, T, width, ldx, nb, inv, codes, scale);
  return cudaGetLastError();
}

cudaError_t launch_checkpoint_restore(const int8_t* codes, const float* scale, long long T, int width, void* out,
                                      int is_bf16, long long ldo, cudaStream_t stream) {
  const int nb = (width + BLOCK - 1) / BLOCK;
  uint32_t inv;
  const unsigned ctas = plan_pairs(T, nb, &inv);
  if (is_bf16)
    checkpoint_restore_kernel<true><<<ctas, THREADS, 0, stream>>>(codes, scale, T, width, nb, inv, out, ldo);
  else
    checkpoint_restore_kernel<false><<<ctas, THREADS, 0, stream>>>(codes, scale, T, width, nb, inv, out, ldo);
  return cudaGetLastError();
}

}  // namespace admmq
