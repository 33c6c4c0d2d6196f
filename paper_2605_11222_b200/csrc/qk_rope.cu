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
// slices of heads instead.  Forward a thread loads two heads (bf16) at once: 63 us for 16384 rows of 40 heads of 128, 83 % of
// the copy rate.  Backward the grid is the resident one: a thread sums the weight's gradient over all its rows in 16
// registers, the CTA's sums go to a workspace, and a second launch adds them in a fixed order.  That leaves few warps, so
// what a thread needs next, up to DEPTH heads ahead and across rows, is on its way into slots of shared memory of its
// own (asynchronous copies: no registers, no barrier); with loads into registers 8192 rows took 58 us, so 55.  What bounds
// it there is latency with 16 warps a multiprocessor (128 registers a thread): DRAM is 50 % busy, issue slots 60 %.
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
// 8 values into this thread's slots: 16-byte pieces, THREADS slots apart.
template <bool BF16>
__device__ __forceinline__ void copy8(uint32_t slot, const void* base, long long at) {
  const char* p = (const char*)base + at * (BF16 ? 2 : 4);
#pragma unroll
  for (int q = 0; q < (BF16 ? 1 : 2); ++q)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot + q * THREADS * 16), "l"(p + 16 * q) : "memory");
}
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> slot8(const uint4* slot) {
  Raw8<BF16> r;
#pragma unroll
  for (int q = 0; q < (BF16 ? 1 : 2); ++q) r.v[q] = slot[q * THREADS];
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
template <bool BF16, int L, int UNR>
__global__ void __launch_bounds__(THREADS, 3) qk_forward_kernel(const __grid_constant__ QkParams P) {
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
      Raw8<BF16> r0[UNR], r1[UNR];
      bool on[UNR];
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        const int h = h0 + grp + u * step;
        on[u] = held && h < A.heads;
        if (on[u]) {
          const long long at = t * A.x_row + (long long)h * A.x_head;
          r0[u] = load8<BF16>(A.x, at + o0);
          r1[u] = load8<BF16>(A.x, at + o1);
        } else {
          r0[u] = r1[u] = Raw8<BF16>{};
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
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z0 = x0[e] * r * w0[e], z1 = x1[e] * r * w1[e];
          out0[e] = rotated ? z0 * c[e] - z1 * s[e] : z0;
          out1[e] = rotated ? z1 * c[e] + z0 * s[e] : z1;
        }
        if (on[u]) {
          const long long ao = t * A.out_row + (long long)(h0 + grp + u * step) * A.out_head;
          store8<BF16>(A.out, ao + o0, out0);
          store8<BF16>(A.out, ao + o1, out1);
        }
      }
    }
  }
}

constexpr int RESIDENT = 2;                           // CTAs of the gradient that a multiprocessor holds
template <bool BF16>
struct Ahead {
  static constexpr int PIECES = BF16 ? 4 : 8;         // 16-byte pieces of a head that a thread holds: x and dy
  static constexpr int DEPTH = BF16 ? 4 : 2;
  static constexpr int BYTES = DEPTH * PIECES * THREADS * 16;
};

// L threads a head (a power of two; threads past d / 16 hold nothing).
template <bool BF16, int L>
__global__ void __launch_bounds__(THREADS, RESIDENT) qk_backward_kernel(const __grid_constant__ QkParams P) {
  pdl_launch();
  using AH = Ahead<BF16>;
  constexpr int G = 32 / L;                       // heads a warp holds at once
  extern __shared__ uint4 slots[];                // [DEPTH][PIECES][THREADS]
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

  Raw8<BF16> wr0 = {}, wr1 = {};                  // the weight as it lies in memory (bf16: half the registers)
  if (held) {
    wr0 = load8<BF16>(A.w, o0);
    wr1 = load8<BF16>(A.w, o1);
  }
  float gw[16];                                   // sums for the weight's gradient
#pragma unroll
  for (int e = 0; e < 16; ++e) gw[e] = 0.0f;

  // this warp's heads: items (row, slice) it, it + stride, ...; in each slice G + grp + k step.  The position of a walk is
  // the warp's, so that the shuffles agree.
  const long long items = P.T * slices, stride = (long long)blocks * WARPS;
  struct Walk {
    long long it, t;
    int h0;
  };
  auto row_of = [&](Walk& w) {
    w.t = slices == 1 ? w.it : w.it / slices;
    w.h0 = (int)(w.it - w.t * slices) * G;
  };
  auto step_on = [&](Walk& w) -> bool {           // true: at another row
    w.h0 += step;
    if (w.h0 < A.heads) return false;
    w.it += stride;
    row_of(w);
    return true;
  };
  auto ask = [&](const Walk& w, uint32_t stage) {
    if (w.it < items && held && w.h0 + grp < A.heads) {
      const uint32_t slot = (uint32_t)__cvta_generic_to_shared(slots + stage * (AH::PIECES * THREADS) + threadIdx.x);
      const long long at = w.t * A.x_row + (long long)(w.h0 + grp) * A.x_head;
      constexpr int RUN = (BF16 ? 1 : 2) * THREADS * 16;
      copy8<BF16>(slot, A.x, at + o0);
      copy8<BF16>(slot + RUN, A.x, at + o1);
      const long long ad = w.t * A.dy_row + (long long)(w.h0 + grp) * A.dy_head;
      copy8<BF16>(slot + 2 * RUN, A.dy, ad + o0);
      copy8<BF16>(slot + 3 * RUN, A.dy, ad + o1);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  Walk now = {(long long)block * WARPS + warp, 0, 0};
  row_of(now);
  Walk next = now;
#pragma unroll
  for (int k = 0; k < AH::DEPTH - 1; ++k) {
    ask(next, k);
    step_on(next);
  }
  uint32_t stage = 0;
  bool fresh = true;                              // a row whose angles are not here yet
  float c[8], s[8];
  while (now.it < items) {
    ask(next, stage == 0 ? AH::DEPTH - 1 : stage - 1);     // into the slots read last
    step_on(next);
    if (fresh) {
      if (rotated) {
        long long pos = P.pos[now.t];
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
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(AH::DEPTH - 1) : "memory");
    const bool on = held && now.h0 + grp < A.heads;
    const uint4* mine = slots + stage * (AH::PIECES * THREADS) + threadIdx.x;
    constexpr int RUN = (BF16 ? 1 : 2) * THREADS;
    float x0[8], x1[8], out0[8], out1[8], w0[8], w1[8];
    unpack8<BF16>(on ? slot8<BF16>(mine) : Raw8<BF16>{}, x0);
    unpack8<BF16>(on ? slot8<BF16>(mine + RUN) : Raw8<BF16>{}, x1);
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], ss));
    const float r = rsqrtf(fmaf(sum_lanes<L>(ss), P.inv_d, P.eps));
    unpack8<BF16>(wr0, w0);
    unpack8<BF16>(wr1, w1);
    float d0[8], d1[8];
    unpack8<BF16>(on ? slot8<BF16>(mine + 2 * RUN) : Raw8<BF16>{}, d0);
    unpack8<BF16>(on ? slot8<BF16>(mine + 3 * RUN) : Raw8<BF16>{}, d1);
    float dot = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g0 = rotated ? d0[e] * c[e] + d1[e] * s[e] : d0[e];
      const float g1 = rotated ? d1[e] * c[e] - d0[e] * s[e] : d1[e];
      x0[e] *= r;                              // n
      x1[e] *= r;
      if (on) {                                // (an absent head's zeros times r could be 0 * inf)
        gw[e] = fmaf(g0, x0[e], gw[e]);
        gw[8 + e] = fmaf(g1, x1[e], gw[8 + e]);
      }
      d0[e] = g0 * w0[e];                      // dn
      d1[e] = g1 * w1[e];
      dot = fmaf(d0[e], x0[e], fmaf(d1[e], x1[e], dot));
    }
    dot = sum_lanes<L>(held ? dot : 0.0f) * P.inv_d;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      out0[e] = r * (d0[e] - x0[e] * dot);
      out1[e] = r * (d1[e] - x1[e] * dot);
    }
    if (on) {
      const long long ao = now.t * A.out_row + (long long)(now.h0 + grp) * A.out_head;
      store8<BF16>(A.out, ao + o0, out0);
      store8<BF16>(A.out, ao + o1, out1);
    }
    fresh = step_on(now);
    if (++stage == AH::DEPTH) stage = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // this CTA's sums: lanes of equal l within the warp, then the warps in order
  __shared__ float red[WARPS][16 * L];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float v = gw[e];
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

// Weight gradients: the CTAs' partial sums in a fixed order.  One block for 32 values of one part; warp y adds every
// 32nd partial, then the 32 sums are added in order.
template <bool BF16>
__global__ void __launch_bounds__(1024)
qk_weight_grad_kernel(const float* __restrict__ partial, int blocks0, int blocks, int d, void* gq, void* gk) {
  __shared__ float red[32][33];
  pdl_wait();                                     // launched beside the end of the kernel that makes the partial sums
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

template <bool BF16, int L>
cudaError_t launch_l(const QkParams& P, bool backward, int blocks, cudaStream_t stream) {
  if (backward) {
    constexpr int BYTES = Ahead<BF16>::BYTES;
    const cudaError_t e = ensure_dynamic_smem((const void*)qk_backward_kernel<BF16, L>, BYTES);
    if (e != cudaSuccess) return e;
    qk_backward_kernel<BF16, L><<<blocks, THREADS, BYTES, stream>>>(P);
  } else {
    qk_forward_kernel<BF16, L, (BF16 ? 2 : 1)><<<blocks, THREADS, 0, stream>>>(P);
  }
  return cudaGetLastError();
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
  // Forward: whole rows a warp while there are enough rows to give every multiprocessor 16 warps; below that a row is cut,
  // to the point where a thread holds one head.  Backward: at most the resident CTAs, shared out by the number of heads,
  // and rows cut until a warp has a dozen pieces (with four or five whole rows the slowest warp takes a sixth longer than
  // the mean).
  const bool bf = a.dtype == ADMMQ_BF16;
  const int heads[2] = {a.q_heads, a.k_heads};
  long long n[2] = {0, 0};
  for (int q = 0; q < 2; ++q) {
    P.slices[q] = 1;
    if (heads[q] == 0) continue;
    long long cap = 0x3fffffffLL, want = (long long)sms * 16;
    if (backward) {
      const long long ctas = RESIDENT * sms < QK_GRAD_BLOCKS ? RESIDENT * sms : QK_GRAD_BLOCKS;
      cap = ctas * heads[q] / (heads[0] + heads[1]);
      cap = cap < 1 ? 1 : q == 0 && heads[1] > 0 && cap == ctas ? ctas - 1 : cap;
      want = cap * WARPS * 12;
    }
    const int most = (heads[q] + G - 1) / G;
    const long long sl = a.n_rows > 0 ? (want + a.n_rows - 1) / a.n_rows : 1;
    P.slices[q] = (int)(sl > most ? most : sl);
    n[q] = (a.n_rows * P.slices[q] + WARPS - 1) / WARPS;
    if (!backward && n[q] > cap) return cudaErrorInvalidValue;
    n[q] = n[q] < cap ? n[q] : cap;
  }
  P.blocks0 = (int)n[0];
  const long long blocks = n[0] + n[1];
  if (blocks > 0) {
    cudaError_t e = cudaSuccess;
#define QK_CASE(LL)                                                                                                   \
  case LL:                                                                                                            \
    e = bf ? launch_l<true, LL>(P, backward, (int)blocks, stream) : launch_l<false, LL>(P, backward, (int)blocks, stream);        \
    break;
    switch (L) {
      QK_CASE(1) QK_CASE(2) QK_CASE(4) QK_CASE(8) QK_CASE(16)
    }
#undef QK_CASE
    if (e != cudaSuccess) return e;
  }
  if (backward) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((a.head_dim + 31) / 32, 2);
    cfg.blockDim = dim3(1024);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = blocks > 0 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, bf ? qk_weight_grad_kernel<true> : qk_weight_grad_kernel<false>,
                              (const float*)P.partial, P.blocks0, (int)blocks, a.head_dim, a.d_grad_wq, a.d_grad_wk);
  }
  return cudaGetLastError();
}

}  // namespace admmq
