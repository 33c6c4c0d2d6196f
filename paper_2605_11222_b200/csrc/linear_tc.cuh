// What the two tensor-core forms of the projection share: expansion of packed codes into a shared-memory operand tile,
// descriptors, tensor maps.
#pragma once
#include <atomic>

#include "adapt.h"
#include "tc_ptx.cuh"

namespace admmq {

extern std::atomic<long long> g_linear_wait_limit;   // bound of every device-side wait, cycles
extern std::atomic<int> g_linear_hold_loads;         // tests: the producers issue nothing

constexpr int BK = 64;                               // K step
// Stage of a step's weights as they are stored: 128 runs of 64 codes (32 bytes each), then their 128 (Delta, z0) pairs.
// A run is 64 input channels of one output channel: forward 128 output channels, backward 64 output channels of two
// neighbouring blocks of input channels.
constexpr int RUNS = 128;
constexpr int CODE_BYTES = RUNS * BK / 2, CODE_STAGE_BYTES = CODE_BYTES + RUNS * 8;

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// Plain bulk copy; addresses and size are multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// Tile with the non-contracted index contiguous: two blocks of 64 of its values (8 KB apart), each 64 K rows of 128
// bytes with 128B swizzle; groups of 8 K rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t make_mmajor_sw128_desc(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

// Copies of K step kb for the 128 values from m0 (below the matrix's end, or nothing is copied and the barrier is
// completed all the same).  Runs past the matrix are not copied: read_codes gives them a grid of (0, 0).
template <bool GRAD>
__device__ __forceinline__ void load_codes(const PackedLayer& L, int m0, int kb, uint32_t dst, uint32_t bar) {
  const int p = L.d_out;
  if (!GRAD) {
    const int runs = min(RUNS, p - m0);
    if (runs <= 0) {
      mbar_arrive(bar);
      return;
    }
    mbar_expect_tx(bar, (uint32_t)runs * 40u);
    bulk_load(dst, L.codes + ((long long)kb * p + m0) * BLOCK_WORDS, (uint32_t)runs * 32u, bar);
    bulk_load(dst + CODE_BYTES, L.grid + (long long)(kb * CODE_BLOCK / L.gs) * p + m0, (uint32_t)runs * 8u, bar);
  } else {
    const int runs = min(BK, p - kb * BK), ib = m0 / CODE_BLOCK, blocks = min(2, L.nib - ib);
    if (blocks <= 0) {
      mbar_arrive(bar);
      return;
    }
    mbar_expect_tx(bar, (uint32_t)(blocks * runs) * 40u);
    for (int b = 0; b < blocks; ++b) {
      bulk_load(dst + b * (CODE_BYTES / 2), L.codes + ((long long)(ib + b) * p + kb * BK) * BLOCK_WORDS,
                (uint32_t)runs * 32u, bar);
      bulk_load(dst + CODE_BYTES + b * (RUNS * 4), L.grid + (long long)((ib + b) * CODE_BLOCK / L.gs) * p + kb * BK,
                (uint32_t)runs * 8u, bar);
    }
  }
}

// Bounded waits.  The polling loop is a call: inlined into every role it made the loops of a kernel whose warps run six
// different ones too long for the instruction caches (the issuer's pass over a step, some 60 instructions, took 1000
// cycles).  A wait returns false, with the abort flag and the device status raised, when the limit runs out.
static __device__ __noinline__ bool poll_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                              long long limit) {
  return mbar_wait(bar, parity, abort_flag, status, limit);
}
struct Waiter {
  volatile int* abort_flag;
  int* status;
  long long limit;
  // one thread
  __device__ __forceinline__ bool one(uint32_t bar, uint32_t parity) const {
    if (mbar_try_wait(bar, parity)) return true;
    return poll_slow(bar, parity, abort_flag, status, limit);
  }
  // A whole warp, all lanes polling in one instruction.  The answer is one for the warp: lanes give up by their own clocks,
  // and where the barrier completes just then some would go on to warp-wide instructions that the others never reach.
  __device__ __forceinline__ bool all(uint32_t bar, uint32_t parity) const {
    bool ok = true;
    if (!mbar_try_wait(bar, parity)) ok = poll_slow(bar, parity, abort_flag, status, limit);
    return __all_sync(0xffffffffu, ok) != 0;
  }
};
// Descriptors differ in their low words only (address, and the leading offset of the second form).
__device__ __forceinline__ uint64_t desc_of(uint64_t base, uint32_t bytes) {
  return (base & 0xffffffff00000000ull) | ((uint32_t)base + (bytes >> 4));
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}

// Half a run (unit u = 2 run + half): 32 codes and the run's grid.
struct CodeRun {
  uint4 c;
  float2 grid;
};
template <bool GRAD>
__device__ __forceinline__ CodeRun read_codes(const PackedLayer& L, const uint8_t* stage, int u, int m0, int kb) {
  const int run = u >> 1;
  const bool in = GRAD ? m0 / CODE_BLOCK + (run >> 6) < L.nib && kb * BK + (run & 63) < L.d_out : m0 + run < L.d_out;
  CodeRun r;
  r.c = *reinterpret_cast<const uint4*>(stage + u * 16);
  r.grid = *reinterpret_cast<const float2*>(stage + CODE_BYTES + run * 8);
  if (!in) r.grid = make_float2(0.f, 0.f);           // whatever the codes: weights of zero
  return r;
}

// (Delta, z0) prepared for codes placed in the mantissa of a number in [1, 2): nibble at bit 19: 1 + k / 16, at bit 15:
// 1 + k / 256, so that z0 + Delta k = (z0 - 16 Delta) + 16 Delta (1 + k / 16), one fma.
struct Expand {
  float2 sa, ba, sb, bb;
};
__device__ __forceinline__ Expand expand_of(float2 grid) {
  const float a = 16.0f * grid.x, b = 256.0f * grid.x;
  return {make_float2(a, a), make_float2(grid.y - a, grid.y - a), make_float2(b, b), make_float2(grid.y - b, grid.y - b)};
}
__device__ __forceinline__ uint32_t expand_pair(uint32_t lo, uint32_t hi, uint32_t mask, float2 s, float2 b) {
  const float2 k = make_float2(__uint_as_float((lo & mask) | 0x3f800000u), __uint_as_float((hi & mask) | 0x3f800000u));
  const float2 w = __ffma2_rn(k, s, b);
  return float2_to_bf16x2(w.x, w.y);
}
// One word of codes -> 8 weights.  w holds channels 0 2 4 6 1 3 5 7 from the lowest nibble on; v is w with its halves
// swapped, so that one shift brings a pair of neighbours to the same bit position.  The shifts go left, as
// multiplications: masks, the rotation and the conversions already fill the integer pipe.
__device__ __forceinline__ uint4 expand8(uint32_t w, const Expand& e) {
  const uint32_t v = __byte_perm(w, w, 0x1032);
  const uint32_t w7 = w * 128u, v7 = v * 128u, w15 = w * 32768u, v15 = v * 32768u;
  uint4 o;
  o.x = expand_pair(w15, v15, 0x00078000u, e.sb, e.bb);
  o.y = expand_pair(w15, v15, 0x00780000u, e.sa, e.ba);
  o.z = expand_pair(w7, v7, 0x00078000u, e.sb, e.bb);
  o.w = expand_pair(w7, v7, 0x00780000u, e.sa, e.ba);
  return o;
}
struct Weights32 {
  uint4 w[4];
};
__device__ __forceinline__ Weights32 expand_unit(const CodeRun& r) {
  const Expand e = expand_of(r.grid);
  return {{expand8(r.c.x, e), expand8(r.c.y, e), expand8(r.c.z, e), expand8(r.c.w, e)}};
}
// The 32 weights of unit u into the 128B-swizzled operand tile (a run is a row of 128 bytes).
__device__ __forceinline__ void write_weights(uint8_t* tile, int u, const Weights32& w) {
  uint8_t* dst = tile + (u >> 1) * 128;
  const int sw = (u >> 1) & 7, ch = 4 * (u & 1);
#pragma unroll
  for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(dst + (((ch + e) ^ sw) << 4)) = w.w[e];
}

// Row-major bf16 tensor map; sizes innermost first, strides in bytes; out of range reads as zero.
bool encode_bf16(CUtensorMap* map, const bf16* ptr, int dims, const cuuint64_t* size, const cuuint64_t* stride_bytes,
                 const cuuint32_t* box, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B);

// ---- linear_pair.cu ----
constexpr int PAIR_ROWS = 512, PAIR_VALUES = 256;    // tile of a pair
cudaError_t launch_linear_pair(bool grad, const PackedLayer& L, const AdapterView* ad, long long T,
                               const int* row_adapter, const bf16* x, long long ldx, bf16* y, long long ldy,
                               const float* h, int* status, int sms, cudaStream_t stream);

}  // namespace admmq
