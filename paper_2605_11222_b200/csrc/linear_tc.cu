// The projection and its input gradient for many rows, on the tensor cores straight from the packed codes:
//   forward     y[t][m]  = sum_k x[t][k]  W[m][k] + sum_r h[t][r] up_a[r][m]      (m: output channel, k: input channel)
//   grad_input  dx[t][m] = sum_k dy[t][k] W[k][m] + sum_r u[t][r] down_a[r][m]    (m: input channel, k: output channel)
//
// The product is formed as D[m][t]: weights are the M operand (128 rows of tensor memory), rows the N operand.  A K step
// of 64 takes 128 x 64 weights, which eight warps expand from codes into the 128-byte-swizzled shared-memory tile:
// 128 runs of 64 input channels of one output channel, in both directions -- forward they are 128 output channels
// (K-major operand), backward 64 output channels times two runs (M-major operand); only the descriptors differ.
// Weights are expanded in fp32 (z0 + Delta k, one fma) and rounded once to bf16: the rounding of a weight is random
// over the K terms of a sum and as large as the one rounding of the output.
// The adapters are further K steps of the same accumulation: for every distinct adapter among the tile's rows the M
// operand is the adapter's output side (rank-major, so M-major) and the N operand is h with the rows of other
// adapters zeroed, in bf16.
//
// One CTA per 128 x NT tile, or a cluster of them that split K when there are few tiles: the fp32 partials stay in the
// CTAs' shared memory and every CTA adds up its share of the rows over distributed shared memory, in rank order.
//   warp 0      producer: codes (bulk copies) and rows (tile loads) into a ring of stages
//   warp 1      allocates tensor memory, issues the MMAs
//   warps 2-9   expand codes, write masked h, and move the finished tile out
// Every wait is bounded: on expiry the kernel records ADMMQ_ERR_TIMEOUT, lets its copies and MMAs in flight finish
// (bounded as well), frees tensor memory and returns; CTAs of a cluster meet the same barriers on that path.
#include <atomic>

#include "adapt.h"
#include "tc_ptx.cuh"

namespace admmq {

std::atomic<long long> g_linear_wait_limit{2000000000LL};
std::atomic<int> g_linear_hold_loads{0};

namespace {

constexpr int BM = 128, BK = 64;
constexpr int EXPAND_WARPS = 8;
constexpr int THREADS = 32 * (2 + EXPAND_WARPS);
constexpr int A_BYTES = BM * BK * 2;                 // 16 KB: 128 runs of 64 weights
constexpr int CODE_BYTES = BM * BK / 2;              // 4 KB
constexpr int MAX_SPLIT = 8;

template <int NT>
struct Cfg {
  static constexpr int B_BYTES = NT * BK * 2;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + CODE_BYTES;
  static constexpr int STAGES = NT == 256 ? 4 : NT == 128 ? 6 : 7;
  static constexpr int SUM_BYTES = NT * BM * 4;      // fp32 partial tile, over the stages once they are done
  static constexpr int RING_BYTES = STAGES * STAGE_BYTES > SUM_BYTES ? STAGES * STAGE_BYTES : SUM_BYTES;
  static constexpr int SMEM = RING_BYTES + 1024;
};

struct TcParams {
  CUtensorMap rows;                                  // [T][K] bf16, box NT x 64
  CUtensorMap out_side;                              // [n][rank][M] bf16, box 1 x 64 x 64
  PackedLayer L;
  int M, K, num_kb;
  long long T;
  const int* row_adapter;
  int n_adapters, rank;                              // n_adapters 0: none
  const float* h;
  bf16* y;
  long long ldy;
  int tiles_m;
  int* status;
  long long wait_limit;
  int hold_loads;
};

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
// M-major tile: two blocks of 64 M values (8 KB apart), each 64 K rows of 128 bytes with 128B swizzle; groups of 8 K
// rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t make_mmajor_sw128_desc(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// bf16 operands, fp32 accumulate, M = 128; N rows K-major; weights K-major or M-major.
__host__ __device__ constexpr uint32_t idesc_of(uint32_t n_cols, bool m_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (m_major ? 1u << 15 : 0u) | ((n_cols >> 3) << 17) |
         ((uint32_t)(BM >> 4) << 24);
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
// swapped, so that one shift brings a pair of neighbours to the same bit position.
__device__ __forceinline__ uint4 expand8(uint32_t w, const Expand& e) {
  const uint32_t v = __funnelshift_l(w, w, 16);
  const uint32_t w3 = w << 3, v3 = v << 3, w5 = w >> 5, v5 = v >> 5;
  uint4 o;
  o.x = expand_pair(v3, w3, 0x00780000u, e.sa, e.ba);
  o.y = expand_pair(v5, w5, 0x00078000u, e.sb, e.bb);
  o.z = expand_pair(v5, w5, 0x00780000u, e.sa, e.ba);
  o.w = expand_pair(w3, v3, 0x00078000u, e.sb, e.bb);
  return o;
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
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

template <bool GRAD, int NT>
__global__ void __launch_bounds__(THREADS, 1) linear_tc_kernel(const __grid_constant__ TcParams P) {
  using C = Cfg<NT>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[4 * STAGES + 2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s, n_list;
  __shared__ uint32_t fill_state[2];
  __shared__ int own[NT];                            // adapter of every row of the tile, -1: none
  __shared__ int list[NT];                           // the distinct ones, rising

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &abort_s;
  const int split = (int)cluster_ctarank(), splits = gridDim.x;
  const int tm = blockIdx.y % P.tiles_m;
  const long long t0 = (long long)(blockIdx.y / P.tiles_m) * NT;
  const int m0 = tm * BM;

  // stage barriers: codes landed, rows landed, operands written, stage free again
  const uint32_t codes0 = smem_u32(&bars[0]), rows0 = codes0 + 8 * STAGES, ready0 = rows0 + 8 * STAGES;
  const uint32_t empty0 = ready0 + 8 * STAGES, done_bar = empty0 + 8 * STAGES, drain_bar = done_bar + 8;

  if (threadIdx.x == 0) {
    abort_s = 0;
    fill_state[0] = fill_state[1] = 0u;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(codes0 + 8 * s, 1);
      mbar_init(rows0 + 8 * s, 1);
      mbar_init(ready0 + 8 * s, EXPAND_WARPS);
      mbar_init(empty0 + 8 * s, 1);
    }
    mbar_init(done_bar, 1);
    mbar_init(drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(NT)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int i = threadIdx.x; i < NT; i += THREADS)
    own[i] = P.n_adapters > 0 && t0 + i < P.T ? row_adapter_of(P.row_adapter, t0 + i, P.n_adapters) : -1;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  if (warp == 2) {
    int n = 0;
    for (int last = -1; n < NT;) {
      int a = 0x7fffffff;
      for (int i = lane; i < NT; i += 32) a = own[i] > last ? min(a, own[i]) : a;
      a = __reduce_min_sync(0xffffffffu, a);
      if (a == 0x7fffffff) break;
      last = a;
      if (lane == 0) list[n] = a;
      ++n;
    }
    if (lane == 0) n_list = n;
  }
  __syncthreads();

  // K steps of this CTA: its share of the weights, then its share of the (adapter, 64 ranks) steps
  const int kb0 = P.num_kb * split / splits, kb1 = P.num_kb * (split + 1) / splits;
  const int rank_steps = (P.rank + BK - 1) / BK;
  const int extra = n_list * rank_steps;
  const int ex0 = extra * split / splits, ex1 = extra * (split + 1) / splits;
  const int steps = (kb1 - kb0) + (ex1 - ex0);

  if (warp == 0) {
    // ===================== producer =====================
    if (lane == 0 && !P.hold_loads) {
      uint32_t armed = 0u, par = 0u;
      for (int it = 0; it < steps; ++it) {
        const int s = it % STAGES;
        const uint32_t ph = (uint32_t)(it / STAGES) & 1u;
        if (!mbar_wait(empty0 + 8 * s, ph ^ 1u, abort_flag, P.status, P.wait_limit)) break;
        const uint32_t a_s = ring + s * C::STAGE_BYTES, b_s = a_s + A_BYTES, c_s = b_s + C::B_BYTES;
        const uint32_t cb = codes0 + 8 * s, rb = rows0 + 8 * s;
        armed |= 1u << s;
        par = (par & ~(1u << s)) | (ph << s);
        if (it < kb1 - kb0) {
          const int kb = kb0 + it;
          if (!GRAD) {
            const uint32_t bytes = (uint32_t)min(BM, P.L.d_out - m0) * 32u;
            mbar_expect_tx(cb, bytes);
            bulk_load(c_s, P.L.codes + ((long long)kb * P.L.d_out + m0) * BLOCK_WORDS, bytes, cb);
          } else {
            const uint32_t bytes = (uint32_t)min(BK, P.L.d_out - kb * BK) * 32u;
            const int ib = m0 / CODE_BLOCK;
            const bool two = ib + 1 < P.L.nib;
            mbar_expect_tx(cb, two ? 2u * bytes : bytes);
            bulk_load(c_s, P.L.codes + ((long long)ib * P.L.d_out + kb * BK) * BLOCK_WORDS, bytes, cb);
            if (two)
              bulk_load(c_s + CODE_BYTES / 2, P.L.codes + ((long long)(ib + 1) * P.L.d_out + kb * BK) * BLOCK_WORDS,
                        bytes, cb);
          }
          mbar_expect_tx(rb, C::B_BYTES);
          tma_load_2d(b_s, &P.rows, rb, kb * BK, (int)t0);
        } else {
          const int ex = ex0 + it - (kb1 - kb0);
          const int a = list[ex / rank_steps], r0 = (ex % rank_steps) * BK;
          mbar_arrive(cb);
          mbar_expect_tx(rb, A_BYTES);
          tma_load_3d(a_s, &P.out_side, rb, m0, r0, a);
          tma_load_3d(a_s + A_BYTES / 2, &P.out_side, rb, m0 + 64, r0, a);
        }
      }
      fill_state[0] = armed;
      fill_state[1] = par;
    }
  } else if (warp == 1) {
    // ===================== MMA issuer =====================
    if (lane == 0) {
      bool ok = true;
      for (int it = 0; it < steps; ++it) {
        const int s = it % STAGES;
        const uint32_t ph = (uint32_t)(it / STAGES) & 1u;
        ok = mbar_wait(rows0 + 8 * s, ph, abort_flag, P.status, P.wait_limit) &&
             mbar_wait(ready0 + 8 * s, ph, abort_flag, P.status, P.wait_limit);
        if (!ok) break;
        tc_fence_after();
        const uint32_t a_s = ring + s * C::STAGE_BYTES, b_s = a_s + A_BYTES;
        const uint64_t bd = make_kmajor_sw128_desc(b_s);
        const bool weights = it < kb1 - kb0;
        const bool m_major = GRAD || !weights;
        const uint64_t ad = m_major ? make_mmajor_sw128_desc(a_s) : make_kmajor_sw128_desc(a_s);
        const uint32_t step = m_major ? 2048u >> 4 : 32u >> 4;      // 16 K values: 16 rows of 128 bytes, or 32 bytes
        const uint32_t idesc = idesc_of(NT, m_major);
        int k16 = BK / 16;
        if (!weights) {
          const int r0 = ((ex0 + it - (kb1 - kb0)) % rank_steps) * BK;
          k16 = min(BK, P.rank - r0 + 15) / 16;                     // (ranks past the end are zero in both operands)
        }
        for (int k = 0; k < k16; ++k)
          tc_mma_f16(tmem, ad + (uint64_t)(k * step), bd + (uint64_t)(k * 2), idesc, it > 0 || k > 0);
        tc_commit(empty0 + 8 * s);
      }
      if (ok) tc_commit(done_bar);
    }
  } else {
    // ===================== expanding warps =====================
    const int u = threadIdx.x - 64;                  // 0..255: run u / 2, its half u & 1
    const int run = u >> 1, half = u & 1;
    const uint32_t row_off = (uint32_t)run * 128u;
    bool waited = false;
    // the grid entry of this thread's run at K step kb; (0, 0) for runs past the matrix: weights of zero
    const int ib_run = m0 / CODE_BLOCK + (run >> 6);              // backward: block of input channels
    auto grid_at = [&](int kb) -> float2 {
      int j, grp;
      if (!GRAD) {
        j = m0 + run;
        grp = kb * CODE_BLOCK / P.L.gs;
      } else {
        j = kb * BK + (run & 63);
        grp = ib_run * CODE_BLOCK / P.L.gs;
        if (ib_run >= P.L.nib) return make_float2(0.f, 0.f);
      }
      return j < P.L.d_out ? __ldg(P.L.grid + (long long)grp * P.L.d_out + j) : make_float2(0.f, 0.f);
    };
    float2 gnext = kb0 < kb1 ? grid_at(kb0) : make_float2(0.f, 0.f);
    for (int it = 0; it < steps; ++it) {
      const int s = it % STAGES;
      const uint32_t ph = (uint32_t)(it / STAGES) & 1u;
      const bool weights = it < kb1 - kb0;
      const float2 gcur = gnext;
      if (it + 1 < kb1 - kb0) gnext = grid_at(kb0 + it + 1);
      if (!mbar_wait_warp(codes0 + 8 * s, ph, abort_flag, P.status, P.wait_limit)) break;
      uint8_t* stage = ring_ptr + s * C::STAGE_BYTES;
      if (weights) {
        const uint4 c = *reinterpret_cast<const uint4*>(stage + A_BYTES + C::B_BYTES + u * 16);
        const Expand e = expand_of(gcur);
        uint8_t* dst = stage + row_off;
        const uint32_t sw = run & 7;
        // (codes of a run past the matrix were not loaded: any bits, times a grid of (0, 0))
        *reinterpret_cast<uint4*>(dst + (((4 * half + 0) ^ sw) << 4)) = expand8(c.x, e);
        *reinterpret_cast<uint4*>(dst + (((4 * half + 1) ^ sw) << 4)) = expand8(c.y, e);
        *reinterpret_cast<uint4*>(dst + (((4 * half + 2) ^ sw) << 4)) = expand8(c.z, e);
        *reinterpret_cast<uint4*>(dst + (((4 * half + 3) ^ sw) << 4)) = expand8(c.w, e);
      } else {
        if (!waited) {
          pdl_wait();                                // h is complete from here on
          waited = true;
        }
        const int ex = ex0 + it - (kb1 - kb0);
        const int a = list[ex / rank_steps], r0 = (ex % rank_steps) * BK;
        for (int i = u; i < NT * 8; i += 32 * EXPAND_WARPS) {
          const int t = i >> 3, ch = i & 7, r = r0 + 8 * ch;
          uint4 o = make_uint4(0, 0, 0, 0);
          if (own[t] == a && r < P.rank) {
            const float4* src = reinterpret_cast<const float4*>(P.h + (t0 + t) * P.rank + r);
            const float4 x = src[0], y = src[1];
            o.x = float2_to_bf16x2(x.x, x.y);
            o.y = float2_to_bf16x2(x.z, x.w);
            o.z = float2_to_bf16x2(y.x, y.y);
            o.w = float2_to_bf16x2(y.z, y.w);
          }
          *reinterpret_cast<uint4*>(stage + A_BYTES + t * 128 + ((ch ^ (t & 7)) << 4)) = o;
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor core reads what was just written
      __syncwarp();
      if (lane == 0) mbar_arrive(ready0 + 8 * s);
    }
    if (!waited) pdl_wait();                         // (so that this launch ends after the one it overlaps)
    // ---- the finished tile: tensor memory -> fp32 [t][m] in shared memory, over the stages
    const bool ok = steps == 0 || mbar_wait_warp(done_bar, 0u, abort_flag, P.status, P.wait_limit);
    if (ok && !*abort_flag) {
      tc_fence_after();
      const int q = warp & 3, hc = (warp - 2) >> 2;
      float* sums = reinterpret_cast<float*>(ring_ptr) + q * 32 + lane;
#pragma unroll 1
      for (int c = 0; c < NT / 2; c += 16) {
        const int col = hc * (NT / 2) + c;
        uint32_t v[16];
        if (steps > 0) {
          tc_ld16(tmem + (uint32_t)col + ((uint32_t)(q * 32) << 16), v);
          tc_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(col + e) * BM] = __uint_as_float(v[e]);
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (abort_s) {
    if (threadIdx.x == 0) {
      const uint32_t armed = fill_state[0], par = fill_state[1];
      for (int s = 0; s < STAGES; ++s)
        if (armed >> s & 1u) {
          mbar_wait_quiet(codes0 + 8 * s, par >> s & 1u);
          mbar_wait_quiet(rows0 + 8 * s, par >> s & 1u);
        }
    }
    if (threadIdx.x == 32) {
      tc_commit(drain_bar);
      mbar_wait_quiet(drain_bar, 0u);
    }
    __syncthreads();
  }
  if (splits > 1) cluster_sync_all();
  if (!abort_s) {
    // ---- rows of this CTA's share: a warp a row, 4 values a lane, summed over the cluster in rank order
    const int r0 = NT * split / splits, r1 = NT * (split + 1) / splits;
    const int m = m0 + 4 * lane;
    for (int r = r0 + warp; r < r1; r += THREADS / 32) {
      if (t0 + r >= P.T) break;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < splits; ++k) {
        const float4 w = ld_cluster_f4(map_to_cta(ring + (uint32_t)(r * BM + 4 * lane) * 4u, (uint32_t)k));
        v.x += w.x;
        v.y += w.y;
        v.z += w.z;
        v.w += w.w;
      }
      if (m < P.M)                                   // M is a multiple of 8
        *reinterpret_cast<uint2*>(P.y + (t0 + r) * P.ldy + m) =
            make_uint2(float2_to_bf16x2(v.x, v.y), float2_to_bf16x2(v.z, v.w));
    }
  }
  if (splits > 1) cluster_sync_all();                // no CTA leaves while its partial is read
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(NT) : "memory");
  }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
                   q == cudaDriverEntryPointSuccess
               ? (EncodeTiledFn)p
               : (EncodeTiledFn) nullptr;
  }();
  return fn;
}
bool encode(CUtensorMap* map, const bf16* ptr, int dims, const cuuint64_t* size, const cuuint64_t* stride_bytes,
            const cuuint32_t* box) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t one[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)dims, (void*)ptr, size, stride_bytes, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool GRAD, int NT>
cudaError_t launch(TcParams& P, const bf16* x, long long ldx, const AdapterView* ad, int splits, cudaStream_t stream) {
  using C = Cfg<NT>;
  const cuuint64_t xs[2] = {(cuuint64_t)P.K, (cuuint64_t)P.T}, xst[1] = {(cuuint64_t)ldx * 2};
  const cuuint32_t xb[2] = {BK, NT};
  if (!encode(&P.rows, x, 2, xs, xst, xb)) return cudaErrorInvalidValue;
  if (ad) {
    const cuuint64_t as[3] = {(cuuint64_t)P.M, (cuuint64_t)ad->rank, (cuuint64_t)ad->n};
    const cuuint64_t ast[2] = {(cuuint64_t)P.M * 2, (cuuint64_t)P.M * 2 * ad->rank};
    const cuuint32_t ab[3] = {64, BK, 1};
    if (!encode(&P.out_side, ad->out, 3, as, ast, ab)) return cudaErrorInvalidValue;
  }
  const auto kernel = linear_tc_kernel<GRAD, NT>;
  cudaError_t e = ensure_dynamic_smem((const void*)kernel, C::SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(splits, (unsigned)(P.tiles_m * ((P.T + NT - 1) / NT)));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ad ? 2 : 1;                         // with adapters it may start beside the shrink launch before it
  return cudaLaunchKernelEx(&cfg, kernel, P);
}

template <bool GRAD>
cudaError_t dispatch(TcParams& P, const bf16* x, long long ldx, const AdapterView* ad, int sms, cudaStream_t stream) {
  const int nt = P.T <= 64 ? 64 : P.T <= 128 ? 128 : 256;
  const long long tiles = (long long)P.tiles_m * ((P.T + nt - 1) / nt);
  if (tiles > 65535) return cudaErrorInvalidValue;
  int splits = 1;
  while (2 * splits <= MAX_SPLIT && tiles * 2 * splits <= sms && P.num_kb >= 4 * splits) splits *= 2;
  if (nt == 64) return launch<GRAD, 64>(P, x, ldx, ad, splits, stream);
  if (nt == 128) return launch<GRAD, 128>(P, x, ldx, ad, splits, stream);
  return launch<GRAD, 256>(P, x, ldx, ad, splits, stream);
}

}  // namespace

cudaError_t launch_linear_tc(bool grad, const PackedLayer& L, const AdapterView* ad, long long T,
                             const int* row_adapter, const bf16* x, long long ldx, bf16* y, long long ldy,
                             const float* h, int* status, cudaStream_t stream) {
  TcParams P = {};
  P.L = L;
  P.M = grad ? L.d_in : L.d_out;
  P.K = grad ? L.d_out : L.d_in;
  P.num_kb = (P.K + BK - 1) / BK;
  P.T = T;
  P.row_adapter = row_adapter;
  P.n_adapters = ad ? ad->n : 0;
  P.rank = ad ? ad->rank : 0;
  P.h = h;
  P.y = y;
  P.ldy = ldy;
  P.tiles_m = (P.M + BM - 1) / BM;
  P.status = status;
  P.wait_limit = g_linear_wait_limit.load(std::memory_order_relaxed);
  P.hold_loads = g_linear_hold_loads.load(std::memory_order_relaxed);
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  return grad ? dispatch<true>(P, x, ldx, ad, sms, stream) : dispatch<false>(P, x, ldx, ad, sms, stream);
}

}  // namespace admmq
