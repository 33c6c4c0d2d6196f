// h[t][r] = scale_a sum_k x[t][k] mat_a[r][k], a the adapter of row t, for many rows: on the tensor cores, D[lane][t] with
// the adapters of the tile's rows as the M operand (128 / rank of them stacked in the 128 lanes) and the rows as the N
// operand.  Every row meets every stacked adapter and its own one's lanes are read: the multiplications cost nothing
// here.  A tile with more distinct adapters than fit makes further passes over its rows.  Bound by reading the rows where
// there are many (16384 of 4096: 134 MB in 31 us at rank 16, 4.3 TB/s; 35 us at rank 128), by the chain of a step
// (copies, MMAs, stage free again: some 800 cycles, whatever their size) where there are few; hence 128 channels a step
// (6011 rows of 12288, rank 16: 48 us with 64, 37 with 128).
//
// One CTA per 64 or 128 rows, or a cluster that splits K: the fp32 sums stay in the CTAs' shared memory and every CTA adds
// up its share of the rows over distributed shared memory, in rank order.
//   warp 0  rows (tile loads)     warp 1  MMA issuer; tensor memory     warp 2  adapters (tile loads)
//   warp 3  the distinct adapters of the tile's rows                    all     sums -> shared memory -> h
// Waits are bounded as in the other tensor-core kernels, and CTAs of a cluster meet the same barriers on that path.
#include "linear_tc.cuh"

namespace admmq {
namespace {

constexpr int LANES = 128, WARPS = 8, THREADS = 32 * WARPS, MAX_SPLIT = 8;
constexpr int KS = 2;                                // K blocks of 64 in a step
constexpr int M_BYTES = LANES * BK * 2;

template <int ROWS>
struct Cfg {
  static constexpr int X_BYTES = ROWS * BK * 2, STAGE_BYTES = KS * (M_BYTES + X_BYTES);
  // stages of a CTA that has a multiprocessor to itself, and of one that shares it
  static constexpr int ST_MAX = ROWS == 64 ? 4 : 3, ST_MIN = ROWS == 64 ? 2 : 1;
  static constexpr int smem(int stages) { return stages * STAGE_BYTES + 1024; }
  static_assert(ROWS * LANES * 4 <= ST_MIN * STAGE_BYTES, "the sums lie over the stages");
  static_assert(smem(ST_MAX) <= 227 * 1024 - 2048 && smem(ST_MIN) <= 113 * 1024 - 2048, "shared memory");
};

struct ShrinkTcParams {
  CUtensorMap rows;                                  // [T][K] bf16, box 64 x ROWS
  CUtensorMap mat;                                   // [n][rank][K] bf16, box 64 x rank x 1
  const int* row_adapter;
  const float* scale;
  float* h;                                          // [T][rank]
  long long T;
  int n, rank, num_kb, splits, stages;
  int* status;
  long long wait_limit;
  int hold_loads;
};

// bf16 operands, fp32 accumulate, both K-major
__host__ __device__ constexpr uint32_t idesc_of(uint32_t rows) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((rows >> 3) << 17) | ((uint32_t)(LANES >> 4) << 24);
}

template <int ROWS>
__global__ void __launch_bounds__(THREADS, 2) shrink_tc_kernel(const __grid_constant__ ShrinkTcParams P) {
  using C = Cfg<ROWS>;
  constexpr int X_BYTES = C::X_BYTES, STAGE_BYTES = C::STAGE_BYTES;
  pdl_launch();
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * C::ST_MAX + 2];
  __shared__ uint32_t tmem_slot, fill_state[4];
  __shared__ int abort_s, n_list;
  __shared__ int own[ROWS];                          // adapter of every row of the tile, -1: none
  __shared__ int list[ROWS];                         // the distinct ones, rising

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Waiter wait = {&abort_s, P.status, P.wait_limit};
  const int split = (int)cluster_ctarank(), splits = P.splits;
  const long long t0 = (long long)((int)blockIdx.x / splits) * ROWS;
  const int kb0 = P.num_kb * split / splits, nkb = P.num_kb * (split + 1) / splits - kb0;
  const int cap = LANES / P.rank, ST = P.stages;
  // full: a step's operands are in place (rows, adapters); empty: its MMAs have read them; a pass's sums are complete
  const uint32_t full = smem_u32(&bars[0]), empty = full + 8 * ST, done_bar = empty + 8 * ST, drain_bar = done_bar + 8;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int i = 0; i < 4; ++i) fill_state[i] = 0u;
    for (int s = 0; s < ST; ++s) {
      mbar_init(full + 8 * s, 2);
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(done_bar, 1);
    mbar_init(drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(ROWS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 3) {
    for (int i = lane; i < ROWS; i += 32) own[i] = t0 + i < P.T ? row_adapter_of(P.row_adapter, t0 + i, P.n) : -1;
    __syncwarp();
    int n = 0;
    for (int last = -1; n < ROWS;) {
      int a = 0x7fffffff;
      for (int i = lane; i < ROWS; i += 32) a = own[i] > last ? min(a, own[i]) : a;
      a = __reduce_min_sync(0xffffffffu, a);
      if (a == 0x7fffffff) break;
      last = a;
      if (lane == 0) list[n] = a;
      ++n;
    }
    if (lane == 0) n_list = n;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int nl = n_list, passes = (nl + cap - 1) / cap;
  const int r0 = ROWS * split / splits, r1 = (int)min((long long)(ROWS * (split + 1) / splits), P.T - t0);
  const int quads = P.rank / 4;

  // rows without an adapter
  for (int i = threadIdx.x; i < (r1 - r0) * quads; i += THREADS) {
    const int r = r0 + i / quads;
    if (own[r] < 0) *reinterpret_cast<float4*>(P.h + (t0 + r) * P.rank + 4 * (i % quads)) = make_float4(0.f, 0.f, 0.f, 0.f);
  }

  uint32_t s = 0, ph = 0;                            // the ring goes on from pass to pass
  auto next_stage = [&] {
    if (++s == (uint32_t)ST) {
      s = 0;
      ph ^= 1u;
    }
  };
  bool live = true;                                  // as of the last barrier: the same for all, whoever gives up after it
  for (int pass = 0; pass < passes; ++pass) {
    const int first = pass * cap, na = min(cap, nl - first);
    if (live) {
      if ((warp == 0 || warp == 2) && lane == 0 && !P.hold_loads) {
        uint32_t armed = fill_state[warp], par = fill_state[warp + 1];
        for (int k = 0; k < nkb; ++k) {
          const uint32_t fb = full + 8 * s;
          if (!wait.one(empty + 8 * s, ph ^ 1u)) break;
          armed |= 1u << s;
          par = (par & ~(1u << s)) | (ph << s);
          const uint32_t m_s = ring + s * STAGE_BYTES;
          if (warp == 0) {
            mbar_expect_tx(fb, KS * X_BYTES);
#pragma unroll
            for (int j = 0; j < KS; ++j)
              tma_load_2d(m_s + KS * M_BYTES + j * X_BYTES, &P.rows, fb, ((kb0 + k) * KS + j) * BK, (int)t0);
          } else {
            const uint32_t bytes = (uint32_t)P.rank * BK * 2;
            mbar_expect_tx(fb, (uint32_t)(KS * na) * bytes);
            for (int b = 0; b < na; ++b)
#pragma unroll
              for (int j = 0; j < KS; ++j)
                tma_load_3d(m_s + j * M_BYTES + b * bytes, &P.mat, fb, ((kb0 + k) * KS + j) * BK, 0, list[first + b]);
          }
          next_stage();
        }
        fill_state[warp] = armed;
        fill_state[warp + 1] = par;
      } else if (warp == 1) {
        bool ok = true;
        for (int k = 0; k < nkb; ++k) {
          ok = wait.all(full + 8 * s, ph);
          if (!ok) break;
          tc_fence_after();
          const uint64_t ad = make_kmajor_sw128_desc(ring + s * STAGE_BYTES);
          const uint64_t bd = make_kmajor_sw128_desc(ring + s * STAGE_BYTES + KS * M_BYTES);
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < KS * BK / 16; ++j)
              tc_mma_f16(tmem, desc_of(ad, j / 4 * M_BYTES + j % 4 * 32), desc_of(bd, j / 4 * X_BYTES + j % 4 * 32), idesc_of(ROWS),
                         (uint32_t)(k | j));
            tc_commit(empty + 8 * s);
          }
          __syncwarp();
          next_stage();
        }
        if (ok) {
          if (elect_one()) tc_commit(done_bar);
          __syncwarp();
          wait.all(done_bar, (uint32_t)pass & 1u);
        }
      }
    }
    __syncthreads();                                 // (the other warps sleep here rather than poll beside the loops)
    live = abort_s == 0;                             // (no wait runs from here to the next pass)
    if (live) {
      // ---- sums: tensor memory -> fp32 [t][lane] in shared memory, over the stages
      tc_fence_after();
      const int q = warp & 3;
      float* sums = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw))) + q * 32 + lane;
      if (q * 32 < na * P.rank) {
#pragma unroll 1
        for (int c = (warp >> 2) * (ROWS / 2); c < (warp >> 2) * (ROWS / 2) + ROWS / 2; c += 16) {
          uint32_t w[16];
          tc_ld16(tmem + (uint32_t)c + ((uint32_t)(q * 32) << 16), w);
          tc_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) sums[(c + e) * LANES] = __uint_as_float(w[e]);
        }
      }
      tc_fence_before();
    }
    __syncthreads();
    if (splits > 1) cluster_sync_all();
    if (live) {
      for (int i = threadIdx.x; i < (r1 - r0) * quads; i += THREADS) {
        const int r = r0 + i / quads, a = own[r];
        int slot = 0;
        while (slot < na && list[first + slot] != a) ++slot;
        if (a < 0 || slot == na) continue;
        const uint32_t at = ring + (uint32_t)(r * LANES + slot * P.rank + 4 * (i % quads)) * 4u;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < splits; ++k) {
          const float4 w = ld_cluster_f4(splits == 1 ? at : map_to_cta(at, (uint32_t)k));
          v.x += w.x;
          v.y += w.y;
          v.z += w.z;
          v.w += w.w;
        }
        const float sc = P.scale[a];
        *reinterpret_cast<float4*>(P.h + (t0 + r) * P.rank + 4 * (i % quads)) =
            make_float4(v.x * sc, v.y * sc, v.z * sc, v.w * sc);
      }
    }
    // the next pass's copies, which the async proxy makes, come after every read of the sums
    if (pass + 1 < passes) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (splits > 1) cluster_sync_all();
    else __syncthreads();
    tc_fence_after();
  }
  if (abort_s) {
    if (threadIdx.x == 0) {
      // both loads of a stage count on its barrier; where one never came, the bound of the wait is the time that the
      // other is given
      for (int i = 0; i < 4; i += 2)
        for (int s = 0; s < ST; ++s)
          if (fill_state[i] >> s & 1u) mbar_wait_quiet(full + 8 * s, fill_state[i + 1] >> s & 1u);
    }
    if (threadIdx.x == 32) {
      tc_commit(drain_bar);
      mbar_wait_quiet(drain_bar, 0u);
    }
    __syncthreads();
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(ROWS) : "memory");
}

// Clusters of `splits` CTAs with so many stages that run at once on the current device; 0 on error.
template <int ROWS>
int clusters_at_once(int splits, int stages) {
  using C = Cfg<ROWS>;
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES][MAX_SPLIT + 1][2];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  int n = known[dev][splits][stages == C::ST_MAX].load(std::memory_order_relaxed);
  if (n == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(splits);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = C::smem(stages);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = splits;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, shrink_tc_kernel<ROWS>, &cfg) != cudaSuccess || n < 1) return 0;
    known[dev][splits][stages == C::ST_MAX].store(n, std::memory_order_relaxed);
  }
  return n;
}

template <int ROWS>
cudaError_t launch(const bf16* x, long long ldx, long long T, int K, const AdapterView& ad,
                   const int* row_adapter, float* h, int* status, cudaStream_t stream) {
  using C = Cfg<ROWS>;
  ShrinkTcParams P = {};
  const cuuint64_t xs[2] = {(cuuint64_t)K, (cuuint64_t)T}, xst[1] = {(cuuint64_t)ldx * 2};
  const cuuint32_t xb[2] = {BK, ROWS};
  const cuuint64_t ms[3] = {(cuuint64_t)K, (cuuint64_t)ad.rank, (cuuint64_t)ad.n};
  const cuuint64_t mst[2] = {(cuuint64_t)K * 2, (cuuint64_t)K * 2 * ad.rank};
  const cuuint32_t mb[3] = {BK, (cuuint32_t)ad.rank, 1};
  if (!encode_bf16(&P.rows, x, 2, xs, xst, xb) || !encode_bf16(&P.mat, ad.in, 3, ms, mst, mb)) return cudaErrorInvalidValue;
  P.row_adapter = row_adapter;
  P.scale = ad.scale;
  P.h = h;
  P.T = T;
  P.n = ad.n;
  P.rank = ad.rank;
  P.num_kb = (K + KS * BK - 1) / (KS * BK);
  P.status = status;
  P.wait_limit = g_linear_wait_limit.load(std::memory_order_relaxed);
  P.hold_loads = g_linear_hold_loads.load(std::memory_order_relaxed);
  const cudaError_t e = ensure_dynamic_smem((const void*)shrink_tc_kernel<ROWS>, C::smem(C::ST_MAX));
  if (e != cudaSuccess) return e;
  const long long tiles = (T + ROWS - 1) / ROWS;
  if (tiles * MAX_SPLIT > 0x7fffffffLL) return cudaErrorInvalidValue;
  // A CTA has a multiprocessor to itself while there are enough; K is split while every cluster runs at once and a CTA
  // keeps at least four steps.
  const int stages = tiles <= clusters_at_once<ROWS>(1, C::ST_MAX) ? C::ST_MAX : C::ST_MIN;
  int splits = 1;
  while (2 * splits <= MAX_SPLIT && P.num_kb >= 8 / KS * splits && tiles <= clusters_at_once<ROWS>(2 * splits, stages)) splits *= 2;
  P.stages = stages;
  P.splits = splits;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * splits));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::smem(stages);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, shrink_tc_kernel<ROWS>, P);
}

}  // namespace

cudaError_t launch_shrink_tc(const bf16* x, long long ldx, long long T, int K, const AdapterView& ad,
                             const int* row_adapter, float* h, int* status, cudaStream_t stream) {
  // Rank 128, two adapters, K = 4096: 2048 rows 12.2 us in tiles of 64 rows, 16.1 in tiles of 128; 6011 rows 37.1, 35.6
  // (K = 12288: 85.7, 70.6).
  return T <= 4096 ? launch<64>(x, ldx, T, K, ad, row_adapter, h, status, stream)
                   : launch<128>(x, ldx, T, K, ad, row_adapter, h, status, stream);
}

}  // namespace admmq
