// Shared declarations of the kernels that run and adapt quantized layers (the C ABI of admmq_adapt.h).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/admmq_adapt.h"
#include "common.cuh"

namespace admmq {

using bf16 = __nv_bfloat16;

// Packed layer.  codes: [ceil(d_in / 64)][d_out][8] words; word w of a row holds the codes of input channels
// 64 ib + 8 w + e, e = 0..7, channel e in nibble (e & 1) * 4 + (e >> 1): the mask 0x000F000F after a shift by 4 s then
// leaves channels 2 s and 2 s + 1 in the two halves of a register, the order of a packed 16-bit pair.  Channels past
// d_in hold code 0.  grid: [groups][d_out] of (Delta, z0).
constexpr int CODE_BLOCK = 64;
constexpr int BLOCK_WORDS = CODE_BLOCK / 8;
struct PackedLayer {
  const uint32_t* codes;
  const float2* grid;
  int d_in, d_out, nib, gs;      // nib = ceil(d_in / 64); gs = group size (d_in for one group)
};

// Adapters as one direction of the projection sees them: `in` is contracted with the rows, `out` adds to the output.
struct AdapterView {
  const bf16* in;                // [n][rank][K]
  const bf16* out;               // [n][rank][M]
  const float* scale;
  int n, rank;
};

__device__ __forceinline__ int row_adapter_of(const int* __restrict__ row_adapter, long long t, int n_adapters) {
  const int a = row_adapter[t];
  return (unsigned)a < (unsigned)n_adapters ? a : -1;
}

// The second of two dependent launches may start before the first has finished; everything the first one wrote is
// visible after pdl_wait.  pdl_launch: the dependent may start from here on.
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ uint4 ldg_stream(const void* p) {   // read once: not kept in L1
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
__device__ __forceinline__ float2 bf16x2_to_float2(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ uint32_t float2_to_bf16x2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// D += A B for one 16 x 8 x 16 tile: bf16 operands, fp32 sums.
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

int device_sms();                // multiprocessors of the current device; 0 on error
cudaError_t ensure_dynamic_smem(const void* kernel, int bytes);

// ---- linear_small.cu ----
constexpr int SMALL_ROWS = 16;   // rows up to which linear_small runs
cudaError_t launch_shrink(const bf16* x, long long ldx, long long T, int K, const AdapterView& ad,
                          const int* row_adapter, float* h, int spare, int* status, cudaStream_t stream);
cudaError_t launch_linear_small(const PackedLayer& L, const AdapterView* ad, int T, const int* row_adapter,
                                const bf16* x, long long ldx, bf16* y, long long ldy, const float* h,
                                cudaStream_t stream);
// ---- shrink_tc.cu ----
cudaError_t launch_shrink_tc(const bf16* x, long long ldx, long long T, int K, const AdapterView& ad,
                             const int* row_adapter, float* h, int* status, cudaStream_t stream);
// ---- linear_tc.cu ----
struct TcPlan {
  bool pair;                     // CTA pairs (linear_pair.cu)
  int nt, splits, tiles_m;
  long long ctas;
};
TcPlan plan_linear_tc(bool grad, const PackedLayer& L, long long T, int sms);
cudaError_t launch_linear_tc(bool grad, const PackedLayer& L, const AdapterView* ad, long long T,
                             const int* row_adapter, const bf16* x, long long ldx, bf16* y, long long ldy,
                             const float* h, int* status, cudaStream_t stream);
// ---- adapter_grad.cu ----
cudaError_t launch_adapter_grad(const admmq_adapter_grad_args& a, cudaStream_t stream);
// ---- checkpoint8.cu ----
// Most blocks of a checkpoint: of rows of two blocks or more, 2^31 and their values do not fit a device (180 GB).
constexpr long long CHECKPOINT_MAX_BLOCKS = 0x7fffffffLL;
cudaError_t launch_checkpoint_save(const void* x, int is_bf16, long long T, int width, long long ldx, int8_t* codes,
                                   float* scale, cudaStream_t stream);
cudaError_t launch_checkpoint_restore(const int8_t* codes, const float* scale, long long T, int width, void* out,
                                      int is_bf16, long long ldo, cudaStream_t stream);
// ---- qk_rope.cu ----
constexpr int QK_GRAD_BLOCKS = 1024;   // most blocks of the backward kernel (rows of partial weight gradients)
cudaError_t launch_qk(const admmq_qk_args& a, bool backward, cudaStream_t stream);

}  // namespace admmq
