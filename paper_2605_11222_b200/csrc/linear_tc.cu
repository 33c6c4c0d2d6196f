// The projection and its input gradient for many rows, on the tensor cores straight from the packed codes:
//   forward     y[t][m]  = sum_k x[t][k]  W[m][k] + sum_r h[t][r] up_a[r][m]      (m: output channel, k: input channel)
//   grad_input  dx[t][m] = sum_k dy[t][k] W[k][m] + sum_r u[t][r] down_a[r][m]    (m: input channel, k: output channel)
//
// The product is formed as D[m][t]: weights are the M operand (128 rows of tensor memory), rows the N operand.  A K step
// of 64 takes 128 x 64 weights, which four warps expand from codes into the 128-byte-swizzled shared-memory tile:
// 128 runs of 64 input channels of one output channel, in both directions -- forward they are 128 output channels
// (K-major operand), backward 64 output channels times two runs (M-major operand); only the descriptors differ.
// Weights are expanded in fp32 (z0 + Delta k, one fma) and rounded once to bf16: the rounding of a weight is random
// over the K terms of a sum and as large as the one rounding of the output.
// The adapters are further K steps of the same accumulation: for every distinct adapter among the tile's rows the M
// operand is the adapter's output side (rank-major, so M-major) and the N operand is h with the rows of other
// adapters zeroed, in bf16.
//
// This file: few tiles (linear_pair.cu has the form for many).  One CTA per 128 x NT tile, or a cluster of up to eight
// that split K: the fp32 partials stay in the CTAs' shared memory and every CTA adds up its share of the rows over
// distributed shared memory, in rank order.  A step's latency (copy landed, 64 codes a thread expanded, stores, proxy
// fence, arrival) is several times its issue time, so four groups of four warps expand four steps at once, and codes
// travel in a ring of their own ahead of the rows.
//   warp 0      rows (tile loads), and the adapters' output sides
//   warp 1      MMA issuer; tensor memory
//   warps 2-3   codes and (Delta, z0) pairs (bulk copies), every other step each: a thread takes some 250 cycles to issue a
//               copy, backward there are four a step, and one thread's were its bound (input gradient of 900 rows of
//               4096 -> 4096: 48.6 us with one, 36.2 with two, 37.7 with four)
//   warp 4      the distinct adapters of the tile's rows (5-7: none; a warp reads the quarter of tensor memory that its
//               number modulo 4 names)
//   warps 8-23  expand codes, write masked h, and move the finished tile out
// Every wait is bounded: on expiry the kernel records ADMMQ_ERR_TIMEOUT, lets its copies and MMAs in flight finish
// (bounded as well), frees tensor memory and returns; CTAs of a cluster meet the same barriers on that path.
#include "../../include/admmq_testing.h"
#include "linear_tc.cuh"

namespace admmq {

std::atomic<long long> g_linear_wait_limit{2000000000LL};
std::atomic<int> g_linear_hold_loads{0};

namespace {

constexpr int BM = 128;
constexpr int ROLE_WARPS = 8, FIRST_CODE_WARP = 2, CODE_WARPS = 2;
constexpr int EXPAND_WARPS = 16, GROUPS = 4, GROUP_WARPS = EXPAND_WARPS / GROUPS;
constexpr int WARPS = ROLE_WARPS + EXPAND_WARPS, THREADS = 32 * WARPS;
constexpr int W_BYTES = BM * BK * 2;                 // 16 KB: 128 runs of 64 weights
constexpr int MAX_SPLIT = 8;

template <int NT>
struct Cfg {
  static constexpr int X_BYTES = NT * BK * 2;
  static constexpr int STAGE_BYTES = W_BYTES + X_BYTES;
  static constexpr int STAGES = NT == 256 ? 4 : NT == 128 ? 5 : 6;
  // (a multiple of the groups, and at least as many stages as groups: a group, which sees every fourth step, then knows
  // that the phase before the one it waits for is over)
  static constexpr int CSTAGES = NT == 256 ? 4 : 8;
  static_assert(CSTAGES % GROUPS == 0 && STAGES >= GROUPS, "waits by parity");
  static constexpr int SUM_BYTES = NT * BM * 4;      // fp32 partial tile, over the stages once they are done
  static_assert(SUM_BYTES <= STAGES * STAGE_BYTES, "the partial tile lies over the stages");
  static constexpr int SMEM = STAGES * STAGE_BYTES + CSTAGES * CODE_STAGE_BYTES + 1024;
};

struct TcParams {
  CUtensorMap rows;                                  // [T][K] bf16, box 64 x NT
  CUtensorMap out_side;                              // [n][rank][M] bf16, box 64 x box_rows x 1
  PackedLayer L;
  int M, K, num_kb;
  long long T;
  const int* row_adapter;
  int n_adapters, rank;                              // n_adapters 0: none
  int cap, box_rows;                                 // adapters in one K step, rank rows of one load
  const float* h;
  bf16* y;
  long long ldy;
  int tiles_m, splits;                               // splits: CTAs of a cluster
  int* status;
  long long wait_limit;
  int hold_loads;
};

// bf16 operands, fp32 accumulate, M = 128; N rows K-major; weights K-major or M-major.
__host__ __device__ constexpr uint32_t idesc_of(uint32_t n_cols, bool m_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (m_major ? 1u << 15 : 0u) | ((n_cols >> 3) << 17) |
         ((uint32_t)(BM >> 4) << 24);
}

// Rows r0 <= r < r1 of the finished tile: a warp a row, 4 values a lane, the S partials summed in rank order, their loads
// under way together.  A tile that is not split has eight rows of a warp under way (900 rows of 4096 -> 4096: 36.3 us row
// by row, 34.5); with several rows of a split one the partials' loads get in each other's way (64 rows: 12.5 us, 13.3).
template <int S>
__device__ __forceinline__ void move_out(const TcParams& P, uint32_t sums, long long t0, int r0, int r1, int m0) {
  constexpr int R = S == 1 ? 8 : 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = m0 + 4 * lane;
  for (int r = r0 + warp; r < r1; r += R * WARPS) {
    float4 w[R][S];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i == 0 || r + i * WARPS < r1) {
        const uint32_t at = sums + (uint32_t)((r + i * WARPS) * BM + 4 * lane) * 4u;
#pragma unroll
        for (int k = 0; k < S; ++k) w[i][k] = ld_cluster_f4(S == 1 ? at : map_to_cta(at, (uint32_t)k));
      }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float4 v = w[i][0];
#pragma unroll
      for (int k = 1; k < S; ++k) {
        v.x += w[i][k].x;
        v.y += w[i][k].y;
        v.z += w[i][k].z;
        v.w += w[i][k].w;
      }
      if (r + i * WARPS < r1 && m < P.M)             // M is a multiple of 8
        *reinterpret_cast<uint2*>(P.y + (t0 + r + i * WARPS) * P.ldy + m) =
            make_uint2(float2_to_bf16x2(v.x, v.y), float2_to_bf16x2(v.z, v.w));
    }
  }
}

template <bool GRAD, int NT>
__global__ void __launch_bounds__(THREADS, 1) linear_tc_kernel(const __grid_constant__ TcParams P) {
  using C = Cfg<NT>;
  constexpr int ST = C::STAGES, CS = C::CSTAGES;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * ST + 2 * CS + 3];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s, n_list;
  __shared__ uint32_t fill_state[2 + 2 * CODE_WARPS];
  __shared__ int own[NT];                            // adapter of every row of the tile, -1: none
  __shared__ int list[NT];                           // the distinct ones, rising

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Waiter wait = {&abort_s, P.status, P.wait_limit};
  const int split = (int)cluster_ctarank(), splits = P.splits;
  const int tile = (int)blockIdx.x / splits, tm = tile % P.tiles_m;
  const long long t0 = (long long)(tile / P.tiles_m) * NT;
  const int m0 = tm * BM;

  // full: a step's operands are in place; empty: its MMAs have read them; codes landed, read; the list; the end
  const uint32_t full = smem_u32(&bars[0]), empty = full + 8 * ST;
  const uint32_t c_full = empty + 8 * ST, c_empty = c_full + 8 * CS;
  const uint32_t list_bar = c_empty + 8 * CS, done_bar = list_bar + 8, drain_bar = done_bar + 8;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int i = 0; i < 2 + 2 * CODE_WARPS; ++i) fill_state[i] = 0u;
    for (int s = 0; s < ST; ++s) {
      mbar_init(full + 8 * s, 1 + GROUP_WARPS);        // the producer with its bytes, and the expanding group's warps
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < CS; ++s) {
      mbar_init(c_full + 8 * s, 1);
      mbar_init(c_empty + 8 * s, GROUP_WARPS);
    }
    mbar_init(list_bar, 1);
    mbar_init(done_bar, 1);
    mbar_init(drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(NT)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // K steps of this CTA: its share of the weights, then its share of the adapters' steps
  const int kb0 = P.num_kb * split / splits, nkb = P.num_kb * (split + 1) / splits - kb0;
  const int per = P.rank > BK ? 2 : 1;               // steps of `cap` adapters
  struct Extra {
    int first, count;
  };
  auto extra_of = [&](int n) -> Extra {
    const int all = (n + P.cap - 1) / P.cap * per, a = all * split / splits;
    return {a, all * (split + 1) / splits - a};
  };
  auto wait_list = [&](bool whole_warp, bool& ok) -> int {
    if (P.n_adapters == 0) return 0;
    ok = whole_warp ? wait.all(list_bar, 0u)
                    : wait.one(list_bar, 0u);
    return ok ? n_list : 0;
  };

  if (warp == 0) {
    // ===================== rows =====================
    if (lane == 0 && !P.hold_loads) {
      uint32_t armed = 0u, par = 0u;
      int steps = nkb, nl = 0;
      Extra ex = {0, 0};
      bool ok = true;
      for (int it = 0; it < steps; ++it) {
        const uint32_t s = it % ST, ph = (uint32_t)(it / ST) & 1u;
        ok = wait.one(empty + 8 * s, ph ^ 1u);
        if (!ok) break;
        const uint32_t w_s = ring + s * C::STAGE_BYTES, x_s = w_s + W_BYTES, fb = full + 8 * s;
        armed |= 1u << s;
        par = (par & ~(1u << s)) | (ph << s);
        if (it < nkb) {
          mbar_expect_tx(fb, C::X_BYTES);
          tma_load_2d(x_s, &P.rows, fb, (kb0 + it) * BK, (int)t0);
          if (it == nkb - 1) {                       // now the list is needed
            nl = wait_list(false, ok);
            if (!ok) break;
            ex = extra_of(nl);
            steps = nkb + ex.count;
          }
        } else {
          const int e = ex.first + it - nkb;
          const int first = e / per * P.cap, na = min(P.cap, nl - first), r0 = (e % per) * BK;
          const int box_bytes = P.box_rows * 128;
          // an odd number of boxes of 8 or 24 rows leaves half of a 16-deep MMA step: a box past the last adapter (it
          // reads as zero) fills it
          const int boxes = na + ((na * P.box_rows) % 16 != 0 ? 1 : 0);
          mbar_expect_tx(fb, 2 * boxes * box_bytes);
          for (int b = 0; b < boxes; ++b) {
            const int a = b < na ? list[first + b] : P.n_adapters;
            tma_load_3d(w_s + b * box_bytes, &P.out_side, fb, m0, r0, a);
            tma_load_3d(w_s + W_BYTES / 2 + b * box_bytes, &P.out_side, fb, m0 + 64, r0, a);
          }
        }
      }
      fill_state[0] = armed;
      fill_state[1] = par;
    }
  } else if (warp == 1) {
    // ===================== MMA issuer =====================
    // (the whole warp walks the loop and one elected lane issues: see linear_pair.cu)
    bool ok = true;
    uint32_t s = 0, ph = 0;
    const uint64_t x_desc = make_kmajor_sw128_desc(ring + W_BYTES), wm_desc = make_mmajor_sw128_desc(ring);
    const uint64_t w_desc = GRAD ? wm_desc : make_kmajor_sw128_desc(ring);
    auto next_stage = [&] {
      if (++s == ST) {
        s = 0;
        ph ^= 1u;
      }
    };
    for (int it = 0; it < nkb; ++it) {
      ok = wait.all(full + 8 * s, ph);
      if (!ok) break;
      tc_fence_after();
      const uint64_t ad = desc_of(w_desc, s * C::STAGE_BYTES), bd = desc_of(x_desc, s * C::STAGE_BYTES);
      constexpr uint32_t A_STEP = GRAD ? 2048 : 32;                  // 16 K values: 16 rows of 128 bytes, or 32 bytes
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
          tc_mma_f16(tmem, desc_of(ad, k * A_STEP), desc_of(bd, k * 32), idesc_of(NT, GRAD), k > 0 ? 1u : (uint32_t)it);
        tc_commit(empty + 8 * s);
      }
      __syncwarp();
      next_stage();
    }
    if (ok && P.n_adapters > 0) {
      ok = wait.all(list_bar, 0u);
      const int nl = ok ? n_list : 0;
      const Extra ex = extra_of(nl);
      for (int e = ex.first; e < ex.first + ex.count && ok; ++e) {
        ok = wait.all(full + 8 * s, ph);
        if (!ok) break;
        tc_fence_after();
        const uint64_t ad = desc_of(wm_desc, s * C::STAGE_BYTES), bd = desc_of(x_desc, s * C::STAGE_BYTES);
        const int na = min(P.cap, nl - e / per * P.cap), r0 = (e % per) * BK;
        const int k16 = P.cap > 1 ? (na * P.box_rows + 15) / 16 : (min(BK, P.rank - r0) + 15) / 16;
        if (elect_one()) {
          for (int k = 0; k < k16; ++k)
            tc_mma_f16(tmem, desc_of(ad, k * 2048), desc_of(bd, k * 32), idesc_of(NT, true), 1u);
          tc_commit(empty + 8 * s);
        }
        __syncwarp();
        next_stage();
      }
    }
    if (ok && elect_one()) tc_commit(done_bar);
    __syncwarp();
  } else if (warp >= FIRST_CODE_WARP && warp < FIRST_CODE_WARP + CODE_WARPS) {
    // ===================== codes and grid =====================
    if (lane == 0 && !P.hold_loads) {
      uint32_t armed = 0u, par = 0u;
      for (int it = warp - FIRST_CODE_WARP; it < nkb; it += CODE_WARPS) {
        const uint32_t s = it % CS, ph = (uint32_t)(it / CS) & 1u;
        if (!wait.one(c_empty + 8 * s, ph ^ 1u)) break;
        armed |= 1u << s;
        par = (par & ~(1u << s)) | (ph << s);
        load_codes<GRAD>(P.L, m0, kb0 + it, ring + ST * C::STAGE_BYTES + s * CODE_STAGE_BYTES, c_full + 8 * s);
      }
      fill_state[2 + 2 * (warp - FIRST_CODE_WARP)] = armed;
      fill_state[3 + 2 * (warp - FIRST_CODE_WARP)] = par;
    }
  } else if (warp == 4) {
    // ===================== the tile's adapters =====================
    if (P.n_adapters > 0) {
      for (int i = lane; i < NT; i += 32) own[i] = t0 + i < P.T ? row_adapter_of(P.row_adapter, t0 + i, P.n_adapters) : -1;
      __syncwarp();
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
      __syncwarp();
      if (lane == 0) mbar_arrive(list_bar);
    }
  } else if (warp >= ROLE_WARPS) {
    // ===================== expanding warps =====================
    const int g = (warp - ROLE_WARPS) / GROUP_WARPS;
    const int v = threadIdx.x - 32 * ROLE_WARPS - g * 32 * GROUP_WARPS;     // 0..127 within the group
    uint32_t s = (uint32_t)g, ph = 0, cs = (uint32_t)g, cph = 0;
    bool waited = false, ok = true;
    int nl = 0, steps = nkb;
    Extra ex = {0, 0};
    bool listed = false;
    for (int it = g; ok; it += GROUPS) {
      if (it >= nkb && !listed) {
        listed = true;
        nl = wait_list(true, ok);
        if (!ok) break;
        ex = extra_of(nl);
        steps = nkb + ex.count;
      }
      if (it >= steps) break;
      uint8_t* w_s = ring_ptr + s * C::STAGE_BYTES;
      uint8_t* x_s = w_s + W_BYTES;
      if (it < nkb) {
        ok = wait.all(c_full + 8 * cs, cph);
        if (!ok) break;
        const uint8_t* cst = ring_ptr + ST * C::STAGE_BYTES + cs * CODE_STAGE_BYTES;
        const CodeRun r0 = read_codes<GRAD>(P.L, cst, v, m0, kb0 + it), r1 = read_codes<GRAD>(P.L, cst, v + 128, m0, kb0 + it);
        __syncwarp();
        if (lane == 0) mbar_arrive(c_empty + 8 * cs);
        cs += GROUPS;
        if (cs >= CS) {
          cs -= CS;
          cph ^= 1u;
        }
        const Weights32 e0 = expand_unit(r0), e1 = expand_unit(r1);     // in registers, before the stage is needed
        ok = wait.all(empty + 8 * s, ph ^ 1u);
        if (!ok) break;
        write_weights(w_s, v, e0);
        write_weights(w_s, v + 128, e1);
      } else {
        if (!waited) {
          pdl_wait();                                // h is complete from here on
          waited = true;
        }
        ok = wait.all(empty + 8 * s, ph ^ 1u);
        if (!ok) break;
        const int e = ex.first + it - nkb, slot0 = e / per * P.cap, na = min(P.cap, nl - slot0), r0 = (e % per) * BK;
        for (int i = v; i < NT * 8; i += 32 * GROUP_WARPS) {
          const int t = i >> 3, ch = i & 7;          // row, 8 ranks
          const int slot = P.cap > 1 ? 8 * ch / P.rank : 0, r = P.cap > 1 ? 8 * ch - slot * P.rank : r0 + 8 * ch;
          uint4 o = make_uint4(0, 0, 0, 0);
          if (slot < na && r < P.rank && own[t] == list[slot0 + slot]) {
            const float4* src = reinterpret_cast<const float4*>(P.h + (t0 + t) * P.rank + r);
            const float4 a = src[0], b = src[1];
            o.x = float2_to_bf16x2(a.x, a.y);
            o.y = float2_to_bf16x2(a.z, a.w);
            o.z = float2_to_bf16x2(b.x, b.y);
            o.w = float2_to_bf16x2(b.z, b.w);
          }
          *reinterpret_cast<uint4*>(x_s + t * 128 + ((ch ^ (t & 7)) << 4)) = o;
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor core reads what was just written
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8 * s);
      s += GROUPS;
      if (s >= ST) {
        s -= ST;
        ph ^= 1u;
      }
    }
    if (!waited) pdl_wait();                         // (so that this launch ends after the one it overlaps)
    // ---- the finished tile: tensor memory -> fp32 [t][m] in shared memory, over the stages
    ok = ok && wait.all(done_bar, 0u);
    if (ok) {
      tc_fence_after();
      const int q = warp & 3, cq = (warp - ROLE_WARPS) >> 2;
      float* sums = reinterpret_cast<float*>(ring_ptr) + q * 32 + lane;
#pragma unroll 1
      for (int c = 0; c < NT / 4; c += 16) {
        const int col = cq * (NT / 4) + c;
        uint32_t w[16];
        tc_ld16(tmem + (uint32_t)col + ((uint32_t)(q * 32) << 16), w);
        tc_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(col + e) * BM] = __uint_as_float(w[e]);
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (abort_s) {
    if (threadIdx.x == 0) {
      const uint32_t armed = fill_state[0], par = fill_state[1];
      for (int s = 0; s < ST; ++s)
        if (armed >> s & 1u) mbar_wait_quiet(full + 8 * s, par >> s & 1u);
      for (int i = 2; i < 2 + 2 * CODE_WARPS; i += 2)
        for (int s = 0; s < CS; ++s)
          if (fill_state[i] >> s & 1u) mbar_wait_quiet(c_full + 8 * s, fill_state[i + 1] >> s & 1u);
    }
    if (threadIdx.x == 32) {
      tc_commit(drain_bar);
      mbar_wait_quiet(drain_bar, 0u);
    }
    __syncthreads();
  }
  if (splits > 1) cluster_sync_all();
  if (!abort_s) {
    const int r0 = NT * split / splits, r1 = (int)min((long long)(NT * (split + 1) / splits), P.T - t0);
    if (splits == 1) move_out<1>(P, ring, t0, r0, r1, m0);
    else if (splits == 2) move_out<2>(P, ring, t0, r0, r1, m0);
    else if (splits == 4) move_out<4>(P, ring, t0, r0, r1, m0);
    else move_out<8>(P, ring, t0, r0, r1, m0);
  }
  if (splits > 1) cluster_sync_all();                // no CTA leaves while its partial is read
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(NT) : "memory");
  }
}

// The answer of a whole-warp wait in every lane, on a barrier that is completed 2^21 cycles after the start; the two halves
// of the warp have limits and abort flags of their own.
__global__ void warp_wait_kernel(long long limit_low, long long limit_high, int* out, int* status) {
  __shared__ __align__(8) uint64_t bar_s;
  __shared__ int flags[2];
  const uint32_t bar = smem_u32(&bar_s);
  const int half = (threadIdx.x & 31) >> 4;
  if (threadIdx.x < 2) flags[threadIdx.x] = 0;
  if (threadIdx.x == 0) mbar_init(bar, 1);
  __syncthreads();
  if (threadIdx.x < 32) {
    const Waiter wait = {&flags[half], status, half ? limit_high : limit_low};
    out[threadIdx.x] = wait.all(bar, 0u) ? 1 : 0;
  } else if (threadIdx.x == 32) {
    const long long t0 = clock64();
    while (clock64() - t0 < (1LL << 21)) {
    }
    mbar_arrive(bar);
  }
  __syncthreads();
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
}  // namespace

bool encode_bf16(CUtensorMap* map, const bf16* ptr, int dims, const cuuint64_t* size, const cuuint64_t* stride_bytes,
                 const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t one[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)dims, (void*)ptr, size, stride_bytes, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <bool GRAD, int NT>
cudaError_t launch(TcParams& P, const bf16* x, long long ldx, const AdapterView* ad, int splits, cudaStream_t stream) {
  using C = Cfg<NT>;
  const cuuint64_t xs[2] = {(cuuint64_t)P.K, (cuuint64_t)P.T}, xst[1] = {(cuuint64_t)ldx * 2};
  const cuuint32_t xb[2] = {BK, NT};
  if (!encode_bf16(&P.rows, x, 2, xs, xst, xb)) return cudaErrorInvalidValue;
  P.cap = P.box_rows = 1;
  if (ad) {
    const cuuint64_t as[3] = {(cuuint64_t)P.M, (cuuint64_t)ad->rank, (cuuint64_t)ad->n};
    const cuuint64_t ast[2] = {(cuuint64_t)P.M * 2, (cuuint64_t)P.M * 2 * ad->rank};
    P.cap = ad->rank <= BK / 2 ? BK / ad->rank : 1;
    P.box_rows = ad->rank <= BK / 2 ? ad->rank : BK;
    const cuuint32_t ab[3] = {64, (cuuint32_t)P.box_rows, 1};
    if (!encode_bf16(&P.out_side, ad->out, 3, as, ast, ab)) return cudaErrorInvalidValue;
  }
  const auto kernel = linear_tc_kernel<GRAD, NT>;
  cudaError_t e = ensure_dynamic_smem((const void*)kernel, C::SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  P.splits = splits;
  cfg.gridDim = dim3((unsigned)(P.tiles_m * ((P.T + NT - 1) / NT) * splits));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  // with adapters it may start beside the shrink launch before it; a cluster only where K is split
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  cfg.numAttrs = 0;
  if (splits > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = splits;
    attr[cfg.numAttrs].val.clusterDim.y = 1;
    attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (ad) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  return cudaLaunchKernelEx(&cfg, kernel, P);
}

// Clusters of `splits` CTAs that run at once on the current device (a multiprocessor holds one CTA in every form); 0 on
// error.  A cluster lies within one group of multiprocessors, and the groups' sizes are not multiples of its own.
int clusters_at_once(int splits) {
  static_assert(Cfg<64>::SMEM > 116 * 1024 && Cfg<128>::SMEM > 116 * 1024, "one CTA a multiprocessor");
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES][MAX_SPLIT + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  int n = known[dev][splits].load(std::memory_order_relaxed);
  if (n == 0) {
    const auto kernel = linear_tc_kernel<false, 256>;
    if (ensure_dynamic_smem((const void*)kernel, Cfg<256>::SMEM) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(splits);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Cfg<256>::SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = splits;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) return 0;
    known[dev][splits].store(n, std::memory_order_relaxed);
  }
  return n;
}

template <bool GRAD>
cudaError_t dispatch(TcParams& P, const bf16* x, long long ldx, const AdapterView* ad, int nt, int splits,
                     cudaStream_t stream) {
  if (P.tiles_m * ((P.T + nt - 1) / nt) * splits > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (nt == 64) return launch<GRAD, 64>(P, x, ldx, ad, splits, stream);
  if (nt == 128) return launch<GRAD, 128>(P, x, ldx, ad, splits, stream);
  return launch<GRAD, 256>(P, x, ldx, ad, splits, stream);
}

}  // namespace

// Form, tile and number of CTAs of a call.
TcPlan plan_linear_tc(bool grad, const PackedLayer& L, long long T, int sms) {
  const int M = grad ? L.d_in : L.d_out, num_kb = ((grad ? L.d_out : L.d_in) + BK - 1) / BK;
  TcPlan p = {};
  p.tiles_m = (M + BM - 1) / BM;
  // Which form: the K steps that the busiest multiprocessor makes, with a step's time in each form (measured: 0.50 us in
  // one CTA on 256 rows, 0.75 us in a pair on 512).  4096 -> 4096: 2048 rows 63 us in single CTAs, 51 in pairs; 900 rows
  // 34 and 48.  333 rows of 1024 -> 4096: 12.5 us in single CTAs that split K, 21 in pairs.
  p.nt = T <= 64 ? 64 : T <= 128 ? 128 : 256;
  const long long tiles = (long long)p.tiles_m * ((T + p.nt - 1) / p.nt);
  const long long pair_tiles = (long long)((M + PAIR_VALUES - 1) / PAIR_VALUES) * ((T + PAIR_ROWS - 1) / PAIR_ROWS);
  // K is split while every cluster runs at once: sixteen clusters of eight do not (333 rows of 4096 -> 1024: 23.1 us in
  // eight parts and two turns, 16.8 in four).
  p.splits = 1;
  while (2 * p.splits <= MAX_SPLIT && num_kb >= 4 * p.splits && tiles * 2 * p.splits <= sms &&
         tiles <= clusters_at_once(2 * p.splits))
    p.splits *= 2;
  const long long single = (tiles * p.splits + sms - 1) / sms * ((num_kb + p.splits - 1) / p.splits);
  const long long pair = (2 * pair_tiles + sms - 1) / sms * num_kb;
  p.pair = 3 * pair < 2 * single;
  p.ctas = p.pair ? sms : tiles * p.splits;
  return p;
}

cudaError_t launch_linear_tc(bool grad, const PackedLayer& L, const AdapterView* ad, long long T,
                             const int* row_adapter, const bf16* x, long long ldx, bf16* y, long long ldy,
                             const float* h, int* status, cudaStream_t stream) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const TcPlan plan = plan_linear_tc(grad, L, T, sms);
  if (plan.pair) return launch_linear_pair(grad, L, ad, T, row_adapter, x, ldx, y, ldy, h, status, sms, stream);
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
  P.status = status;
  P.wait_limit = g_linear_wait_limit.load(std::memory_order_relaxed);
  P.hold_loads = g_linear_hold_loads.load(std::memory_order_relaxed);
  P.tiles_m = plan.tiles_m;
  return grad ? dispatch<true>(P, x, ldx, ad, plan.nt, plan.splits, stream)
              : dispatch<false>(P, x, ldx, ad, plan.nt, plan.splits, stream);
}

}  // namespace admmq

extern "C" admmq_status admmq_test_warp_wait(long long limit_low, long long limit_high, int* d_out, int* d_status,
                                             void* cuda_stream) {
  if (limit_low < 1000 || limit_high < 1000 || limit_low > 2000000000LL || limit_high > 2000000000LL || !d_out || !d_status)
    return ADMMQ_ERR_INVALID_ARG;
  admmq::warp_wait_kernel<<<1, 64, 0, (cudaStream_t)cuda_stream>>>(limit_low, limit_high, d_out, d_status);
  return cudaGetLastError() == cudaSuccess ? ADMMQ_OK : ADMMQ_ERR_CUDA;
}
