// Per-head norm of queries and keys with the position rotation, and its gradient.
//
// With x one head's values, r = 1 / sqrt(mean(x^2) + eps), n = x r, z = w n, y = R z (R: the rotation of the pairs
// (i, i + rot/2) by the position's angles).  Gradient: g = R^T dy, dw = sum g n, dn = g w,
//   dx = r (dn - n mean(dn n)).
//
// Bound: memory, one read and one write of every value (backward: two reads, one write).  A head of 16 L values is
// held by L threads, 16 values each in two runs of 8: run 0 and run 1 of a rotated thread are the two halves of its
// pairs, so the rotation needs no exchange, every access is 16 bytes wide, and the sums are log2(L) shuffles away.
// A CTA works on queries or on keys; one of its warps takes one row (token) at a time and 32 / L of its heads at once,
// so that the weight stays in registers throughout and the rotation's cos and sin for a row.  Few rows are cut into
// slices of heads instead.  The backward kernel's grid is the resident one: a thread sums the weight's gradient over
// all its rows in 16 registers, the CTA's sums go to a workspace, and a second launch adds them in a fixed order.
#include "adapt.h"

namespace admmq {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

struct Part {                    // queries or keys
  const void* x;
  const void* w;
  void* out;
  const void* dy;
  long long x_row, x_head, out_row, out_head, dy_row, dy_head;
  int heads;
};
struct QkParams {
  Part part[2];
  int slices[2];                 // pieces a row's heads are cut into
  int blocks0;                   // CTAs of part 0; the rest work on part 1
  const float* cos;
  const float* sin;
  const int* pos;
  long long T, n_positions;
  float eps, inv_d;
  int d, rot;
  float* partial;                // backward: [blocks][d]
  int* status;
};

template <bool BF16>
struct Raw8 {                    // 8 values as they lie in memory
  uint4 v[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load8(const void* base, long long at) {
  Raw8<BF16> r;
  const char* p = (const char*)base + at * (BF16 ? 2 : 4);
#pragma unroll
  for (int q = 0; q < (BF16 ? 1 : 2); ++q) r.v[q] = *reinterpret_cast<const uint4*>(p + 16 * q);
  return r;
}
template <bool BF16>
__device__ __forceinline__ void unpack8(const Raw8<BF16>& r, float (&f)[8]) {
  if (BF16) {
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 t = bf16x2_to_float2(w[e]);
      f[2 * e] = t.x;
      f[2 * e + 1] = t.y;
    }
  } else {
    const uint4 a = r.v[0], b = r.v[BF16 ? 0 : 1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* base, long long at, const float (&f)[8]) {
  char* p = (char*)base + at * (BF16 ? 2 : 4);
  if (BF16) {
    uint4 o;
    o.x = float2_to_bf16x2(f[0], f[1]);
    o.y = float2_to_bf16x2(f[2], f[3]);
    o.z = float2_to_bf16x2(f[4], f[5]);
    o.w = float2_to_bf16x2(f[6], f[7]);
    *reinterpret_cast<uint4*>(p) = o;
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 16) = make_float4(f[4], f[5], f[6], f[7]);
  }
}
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// L threads a head (a power of two; threads past d / 16 hold nothing), UNR heads of a thread in flight.
template <bool BF16, bool BWD, int L, int UNR>
__global__ void __launch_bounds__(THREADS, BWD ? 2 : 3) qk_kernel(const __grid_constant__ QkParams P) {
  constexpr int G = 32 / L;                       // heads a warp holds at once
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int l = lane % L, grp = lane / L;
  const bool held = l * 16 < P.d;
  const int nrot = P.rot >> 4;
  const bool rotated = l < nrot;
  // runs of 8 values: the halves of the rotated pairs, or 16 consecutive values past the rotated part
  const int o0 = rotated ? 8 * l : P.rot + 16 * (l - nrot);
  const int o1 = rotated ? (P.rot >> 1) + 8 * l : o0 + 8;
  const bool second = (int)blockIdx.x >= P.blocks0;
  const Part& A = P.part[second ? 1 : 0];
  const int slices = P.slices[second ? 1 : 0];
  const int block = second ? blockIdx.x - P.blocks0 : blockIdx.x;
  const int blocks = second ? gridDim.x - P.blocks0 : P.blocks0;
  const int step = G * slices;

  float w0[8], w1[8];
  if (held) {
    unpack8<BF16>(load8<BF16>(A.w, o0), w0);
    unpack8<BF16>(load8<BF16>(A.w, o1), w1);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w0[e] = w1[e] = 0.0f;
  }
  float gw[BWD ? 16 : 1];                         // sums for the weight's gradient
  if (BWD) {
#pragma unroll
    for (int e = 0; e < 16; ++e) gw[BWD ? e : 0] = 0.0f;
  }

  const long long items = P.T * slices;
  for (long long it = (long long)block * WARPS + warp; it < items; it += (long long)blocks * WARPS) {
    const long long t = slices == 1 ? it : it / slices;
    const int slice = (int)(it - t * slices);
    float c[8], s[8];
    if (rotated) {
      long long pos = P.pos[t];
      if ((unsigned long long)pos >= (unsigned long long)P.n_positions) {
        raise_status(P.status, ADMMQ_ERR_SHAPE);
        pos = 0;
      }
      const float4* pc = reinterpret_cast<const float4*>(P.cos + pos * (P.rot >> 1) + 8 * l);
      const float4* ps = reinterpret_cast<const float4*>(P.sin + pos * (P.rot >> 1) + 8 * l);
      const float4 c0 = __ldg(pc), c1 = __ldg(pc + 1), s0 = __ldg(ps), s1 = __ldg(ps + 1);
      c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
      s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = 1.0f;
        s[e] = 0.0f;
      }
    }
    // heads of this thread: slice G + grp + k step; the loop count is the warp's, so that the shuffles agree
    for (int h0 = slice * G; h0 < A.heads; h0 += UNR * step) {
      Raw8<BF16> r0[UNR], r1[UNR], y0[BWD ? UNR : 1], y1[BWD ? UNR : 1];
      bool on[UNR];
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        const int h = h0 + grp + u * step;
        on[u] = held && h < A.heads;
        if (on[u]) {
          const long long at = t * A.x_row + (long long)h * A.x_head;
          r0[u] = load8<BF16>(A.x, at + o0);
          r1[u] = load8<BF16>(A.x, at + o1);
          if (BWD) {
            const long long ad = t * A.dy_row + (long long)h * A.dy_head;
            y0[BWD ? u : 0] = load8<BF16>(A.dy, ad + o0);
            y1[BWD ? u : 0] = load8<BF16>(A.dy, ad + o1);
          }
        } else {
          r0[u] = r1[u] = Raw8<BF16>{};
          if (BWD) y0[BWD ? u : 0] = y1[BWD ? u : 0] = Raw8<BF16>{};
        }
      }
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        float x0[8], x1[8];
        unpack8<BF16>(r0[u], x0);
        unpack8<BF16>(r1[u], x1);
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], ss));
        const float r = rsqrtf(fmaf(sum_lanes<L>(ss), P.inv_d, P.eps));
        float out0[8], out1[8];
        if (!BWD) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z0 = x0[e] * r * w0[e], z1 = x1[e] * r * w1[e];
            out0[e] = rotated ? z0 * c[e] - z1 * s[e] : z0;
            out1[e] = rotated ? z1 * c[e] + z0 * s[e] : z1;
          }
        } else {
          float d0[8], d1[8];
          unpack8<BF16>(y0[BWD ? u : 0], d0);
          unpack8<BF16>(y1[BWD ? u : 0], d1);
          float dot = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float g0 = rotated ? d0[e] * c[e] + d1[e] * s[e] : d0[e];
            const float g1 = rotated ? d1[e] * c[e] - d0[e] * s[e] : d1[e];
            x0[e] *= r;                          // n
            x1[e] *= r;
            if (on[u]) {                         // (an absent head's zeros times r could be 0 * inf)
              gw[BWD ? e : 0] = fmaf(g0, x0[e], gw[BWD ? e : 0]);
              gw[BWD ? 8 + e : 0] = fmaf(g1, x1[e], gw[BWD ? 8 + e : 0]);
            }
            d0[e] = g0 * w0[e];                  // dn
            d1[e] = g1 * w1[e];
            dot = fmaf(d0[e], x0[e], fmaf(d1[e], x1[e], dot));
          }
          dot = sum_lanes<L>(held ? dot : 0.0f) * P.inv_d;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            out0[e] = r * (d0[e] - x0[e] * dot);
            out1[e] = r * (d1[e] - x1[e] * dot);
          }
        }
        if (on[u]) {
          const long long ao = t * A.out_row + (long long)(h0 + grp + u * step) * A.out_head;
          store8<BF16>(A.out, ao + o0, out0);
          store8<BF16>(A.out, ao + o1, out1);
        }
      }
    }
  }

  if (BWD) {
    // this CTA's sums: lanes of equal l within the warp, then the warps in order
    __shared__ float red[WARPS][16 * L];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = gw[BWD ? e : 0];
#pragma unroll
      for (int o = L; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (grp == 0 && held) red[warp][(e < 8 ? o0 : o1) + (e & 7)] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < P.d; i += THREADS) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) v += red[w][i];
      P.partial[(long long)blockIdx.x * P.d + i] = v;
    }
  }
}

// Weight gradients: the CTAs' partial sums in a fixed order.  One block for 32 values of one part; warp y adds every
// 32nd partial, then the 32 sums are added in order.
template <bool BF16>
__global__ void __launch_bounds__(1024)
qk_weight_grad_kernel(const float* __restrict__ partial, int blocks0, int blocks, int d, void* gq, void* gk) {
  __shared__ float red[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + tx, q = blockIdx.y;
  const int b0 = q == 0 ? 0 : blocks0, b1 = q == 0 ? blocks0 : blocks;
  float v = 0.0f;
  if (i < d) {
#pragma unroll 8
    for (int b = b0 + ty; b < b1; b += 32) v += partial[(long long)b * d + i];
  }
  red[ty][tx] = v;
  __syncthreads();
  if (ty == 0 && i < d) {
    v = 0.0f;
#pragma unroll
    for (int y = 0; y < 32; ++y) v += red[y][tx];
    void* g = q == 0 ? gq : gk;
    if (g == nullptr) return;
    if (BF16)
      ((bf16*)g)[i] = __float2bfloat16_rn(v);
    else
      ((float*)g)[i] = v;
  }
}

template <bool BF16, bool BWD, int L>
void launch_l(const QkParams& P, int blocks, cudaStream_t stream) {
  qk_kernel<BF16, BWD, L, (BF16 && !BWD ? 2 : 1)><<<blocks, THREADS, 0, stream>>>(P);
}

}  // namespace

cudaError_t launch_qk(const admmq_qk_args& a, bool backward, cudaStream_t stream) {
  QkParams P = {};
  P.part[0] = {a.d_q, a.d_wq, a.d_out_q, a.d_dy_q, a.q_row, a.q_head, a.out_q_row, a.out_q_head, a.dy_q_row,
               a.dy_q_head, a.q_heads};
  P.part[1] = {a.d_k, a.d_wk, a.d_out_k, a.d_dy_k, a.k_row, a.k_head, a.out_k_row, a.out_k_head, a.dy_k_row,
               a.dy_k_head, a.k_heads};
  P.cos = a.d_cos;
  P.sin = a.d_sin;
  P.pos = a.d_pos;
  P.T = a.n_rows;
  P.n_positions = a.n_positions;
  P.eps = (float)a.eps;
  P.inv_d = 1.0f / (float)a.head_dim;
  P.d = a.head_dim;
  P.rot = a.rot_dim;
  P.partial = (float*)a.d_workspace;
  P.status = a.d_status;
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  int L = 1;
  while (L * 16 < a.head_dim) L *= 2;
  const int G = 32 / L;
  // Whole rows a warp while there are enough rows to give every multiprocessor 16 warps; below that a row is cut, to
  // the point where a thread holds one head.  CTAs: the work's, and for the backward kernel at most the two an SM
  // holds, shared out by the number of heads.
  const long long want = (long long)sms * 16;
  long long n[2] = {0, 0};
  for (int q = 0; q < 2; ++q) {
    const int heads = q == 0 ? a.q_heads : a.k_heads, most = (heads + G - 1) / G;
    const long long sl = a.n_rows > 0 ? (want + a.n_rows - 1) / a.n_rows : 1;
    P.slices[q] = (int)(sl > most ? (most > 0 ? most : 1) : sl);
    n[q] = heads > 0 ? (a.n_rows * P.slices[q] + WARPS - 1) / WARPS : 0;
  }
  if (backward) {
    const int cap = 2 * sms < QK_GRAD_BLOCKS ? 2 * sms : QK_GRAD_BLOCKS, heads = a.q_heads + a.k_heads;
    int c1 = a.k_heads > 0 ? (int)((long long)cap * a.k_heads / heads) : 0;
    if (a.k_heads > 0 && c1 < 1) c1 = 1;
    const int c0 = cap - c1 > 0 ? cap - c1 : 1;
    n[0] = n[0] < c0 ? n[0] : c0;
    n[1] = n[1] < c1 ? n[1] : c1;
  }
  P.blocks0 = (int)n[0];
  const long long blocks = n[0] + n[1];
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  const bool bf = a.dtype == ADMMQ_BF16;
  if (blocks > 0) {
#define QK_CASE(LL)                                                                     \
  case LL:                                                                              \
    if (bf) backward ? launch_l<true, true, LL>(P, (int)blocks, stream) : launch_l<true, false, LL>(P, (int)blocks, stream); \
    else backward ? launch_l<false, true, LL>(P, (int)blocks, stream) : launch_l<false, false, LL>(P, (int)blocks, stream);  \
    break;
    switch (L) {
      QK_CASE(1) QK_CASE(2) QK_CASE(4) QK_CASE(8) QK_CASE(16)
    }
#undef QK_CASE
  }
  if (backward) {
    const dim3 grid((a.head_dim + 31) / 32, 2);
    if (bf)
      qk_weight_grad_kernel<true><<<grid, 1024, 0, stream>>>(P.partial, P.blocks0, (int)blocks, a.head_dim, a.d_grad_wq, a.d_grad_wk);
    else
      qk_weight_grad_kernel<false><<<grid, 1024, 0, stream>>>(P.partial, P.blocks0, (int)blocks, a.head_dim, a.d_grad_wq, a.d_grad_wk);
  }
  return cudaGetLastError();
}

}  // namespace admmq
