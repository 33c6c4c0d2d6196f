// The projection and its input gradient for many rows on pairs of multiprocessors (clusters of two CTAs,
// tcgen05.mma.cta_group::2), straight from the packed codes.  The sums are those of linear_tc.cu.
//
// Tile of a pair: 512 rows by 256 output values.  D[row][value] = sum_k rows[row][k] weights[value][k]: the rows are the
// M operand, two blocks of 256 of which each CTA stages its own 128, the weights the N operand (each CTA expands 128 of
// the 256 values).  So a lane of tensor memory is a row and its columns are neighbours in memory, and one expansion of
// weights serves two MMAs: a K step of 64 takes the tensor cores 1024 cycles and the expansion about 300 issue cycles of
// the four schedulers.  (With one block of rows and alternating accumulators a step took 900 cycles instead of 512,
// measured 894 us against 577 for 8192 rows of 4096 -> 12288.)
//   warp 0       rows (tile loads), and the adapters' output sides; completion of both CTAs' bytes on the leader's barrier
//   warp 1       MMA issuer (leader); tensor memory
//   warp 2       codes and (Delta, z0) pairs (bulk copies) into a ring of their own, further ahead than the rows
//   warp 3       the distinct adapters of the next tile's rows
//   warps 4-7    finished tiles: tensor memory -> registers -> memory
//   warps 8-23   four groups of expanding warps, one K step each in turn, so that a step's latency (copy landed, 64 codes
//                a thread, stores, proxy fence, arrival at the leader) overlaps three others'
// Adapters are further K steps: a step holds as many of the tile's adapters as fit in 64 rank rows; the N operand is
// their output sides, the M operand is h in bf16, zero where a row has another adapter.
// Waits are bounded as in the other tensor-core kernels.  No multicast load anywhere.
// 6011 rows of 4096 -> 4096 without adapters: 153 us, the tensor pipe busy 68 % of the cycles.  192 tiles on 74 pairs are
// 2.6 turns, of which three are paid for, and a tile takes some 17000 cycles beside its 65000 of MMAs (its start, and its way
// out of tensor memory, which one set of accumulators does not overlap).
#include <atomic>

#include "../../include/admmq_testing.h"
#include "linear_tc.cuh"

namespace admmq {
namespace {

constexpr int ROLE_WARPS = 8, EXPAND_WARPS = 16, GROUPS = 4, GROUP_WARPS = EXPAND_WARPS / GROUPS;
constexpr int THREADS = 32 * (ROLE_WARPS + EXPAND_WARPS);
constexpr int HALF = 128;                            // rows and values of a tile that one CTA holds (of 256)
constexpr int X_BYTES = HALF * BK * 2;               // 16 KB a block of rows
constexpr int W_BYTES = HALF * BK * 2;
constexpr int MOVE_WARPS = 4;
constexpr int OUT_COLS = 32, OUT_BUF = 32 * OUT_COLS * 2, OUT_BYTES = 2 * OUT_BUF;   // staging of a moving warp: 2 x 32 rows x 64 bytes
constexpr int NONE = 0xffff;                         // row without an adapter

constexpr int NMB = 2;                               // blocks of 256 rows
struct Cfg {
  // A step's rows are on their way for about 1000 cycles before the MMAs need them, its weights for 2000: rings of
  // different depth.  Barriers go with the weights' ring.
  static constexpr int XST = 3, WST = 5, CST = 4;
  static constexpr int CBARS = 2 * CST;                // barriers of the codes' slots: every slot has two, taken in turn
  static constexpr int W_AT = XST * NMB * X_BYTES, C_AT = W_AT + WST * W_BYTES, OUT_AT = C_AT + CST * CODE_STAGE_BYTES;
  static constexpr int SMEM = OUT_AT + MOVE_WARPS * OUT_BYTES + 1024;
  static constexpr int ROWS = NMB * 256;
};

struct PairParams {
  CUtensorMap rows;                                  // [T][K] bf16, box 64 x 128
  CUtensorMap out_side;                              // [n][rank][M] bf16, box 64 x box_rows x 1
  CUtensorMap out;                                   // [T][M] bf16, box 32 x 32 (stores)
  PackedLayer L;
  int M, K, num_kb;
  long long T;
  const int* row_adapter;
  int n_adapters, rank;                              // n_adapters 0: none
  int cap, box_rows;                                 // adapters in one K step, rank rows of one load
  const float* h;
  int tiles_m, num_tiles;
  int* status;
  long long wait_limit;
  int hold_loads;
};

// Tile load of one CTA of a pair; the bytes are counted by the leader's barrier.
__device__ __forceinline__ void load_pair_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void load_pair_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// Tile store from shared memory; rows and columns past the tensor are left out.
__device__ __forceinline__ void store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x),
               "r"(y)
               : "memory");
}
// Arrives, once the MMAs issued so far are complete, on the barrier at this offset in both CTAs.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile(
      "{\n.reg .b16 m;\nmov.b16 m, 3;\n"
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n}"
      ::"r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// bf16, fp32 accumulate, M = 256 K-major, N = 256 K-major or N-major.
__host__ __device__ constexpr uint32_t idesc_pair(bool n_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (n_major ? 1u << 16 : 0u) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
}

template <bool GRAD>
__global__ void __launch_bounds__(THREADS, 1) linear_pair_kernel(const __grid_constant__ PairParams P) {
  using C = Cfg;
  constexpr int XST = C::XST, WST = C::WST, CS = C::CST, CB = C::CBARS;
  static_assert(WST >= GROUPS && CB % CS == 0 && CB % GROUPS == 0 && CB + 1 >= GROUPS + WST, "see stage_free");
  static_assert(XST <= WST, "a step whose rows' stage is free has its weights' stage free");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * WST + CB + CS + 9];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;
  __shared__ uint32_t fill_state[4];
  __shared__ uint16_t own[2][C::ROWS];               // adapter of every row of the pair's tile
  __shared__ uint16_t list[2][C::ROWS];              // the distinct ones, rising
  __shared__ int list_n[2];

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Waiter wait = {&abort_s, P.status, P.wait_limit};
  const uint32_t rank = cluster_ctarank();           // 0: leader
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const bool adapters = P.n_adapters > 0;

  // full: a step's operands are in place (leader); done: its MMAs have read them (both CTAs); codes landed and read;
  // accumulators complete and moved out; a tile's adapters listed and no longer needed
  const uint32_t full = smem_u32(&bars[0]), done = full + 8 * WST;
  const uint32_t c_full = done + 8 * WST, c_empty = c_full + 8 * CB;
  const uint32_t t_full = c_empty + 8 * CS, t_empty = t_full + 16, l_full = t_empty + 16, l_empty = l_full + 16;
  const uint32_t drain_bar = l_empty + 16;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int i = 0; i < 4; ++i) fill_state[i] = 0u;
    for (int s = 0; s < WST; ++s) {
      // leader's: its producer, expecting the bytes of both CTAs, and the expanding group's warps of both
      mbar_init(full + 8 * s, 1 + 2 * GROUP_WARPS);
      mbar_init(done + 8 * s, 1);
    }
    for (int s = 0; s < CB; ++s) mbar_init(c_full + 8 * s, 1);
    for (int s = 0; s < CS; ++s) mbar_init(c_empty + 8 * s, GROUP_WARPS);
    for (int b = 0; b < 2; ++b) {
      mbar_init(t_full + 8 * b, 1);
      mbar_init(t_empty + 8 * b, 2 * 4);             // leader's: the four moving warps of both CTAs
      mbar_init(l_full + 8 * b, 1);
      mbar_init(l_empty + 8 * b, (rank == 0 ? 2 : 1) + EXPAND_WARPS);
    }
    mbar_init(drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // the peer's barriers exist before any remote arrival
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // a role's view of the adapters of its n-th tile: their number, 0 without waiting if there is no bank
  auto wait_list = [&](uint32_t n, bool whole_warp, bool& ok) -> int {
    if (!adapters) return 0;
    const uint32_t bar = l_full + 8 * (n & 1), ph = (n >> 1) & 1u;
    ok = whole_warp ? wait.all(bar, ph)
                    : wait.one(bar, ph);
    return ok ? list_n[n & 1] : 0;
  };
  // A wait by parity is only sound for a waiter that knows the phase before to be over.  Roles that walk every step know
  // it; an expanding group sees every fourth.  Stages: steps are done in order, so that step it - 4 - WST done (its wait
  // before) covers it - 2 WST, and it - WST done (asked first) covers it - XST - WST.  Codes: they are counted by weights'
  // steps (ct), without the adapters' steps that lie between those of two tiles, so that the group that takes a slot
  // changes from tile to tile.  The phase before that of ct on its barrier is ct - CB.  With no adapter step since then it
  // was this group's own, 8 steps ago; with one or more it was step it - 9 or an earlier one, which step it - 4 - WST done
  // covers.  (One barrier a slot is not enough: ct - 4 may be another group's, and its copy still on the way.)
  // waits until the stage of step `it` in a ring of `depth` stages is free: step it - depth is done
  auto stage_free = [&](uint32_t it, uint32_t depth, bool whole_warp) -> bool {
    if (it < depth) return true;
    const uint32_t last = it - depth, bar = done + 8 * (last % WST), ph = (last / WST) & 1u;
    return whole_warp ? wait.all(bar, ph)
                      : wait.one(bar, ph);
  };
  auto extra_steps = [&](int n) { return (n + P.cap - 1) / P.cap * (P.rank > BK ? 2 : 1); };

  if (warp == 0) {
    // ===================== rows =====================
    if (lane == 0 && !P.hold_loads) {
      uint32_t it = 0, n = 0, armed = 0u, par = 0u;
      bool ok = true;
      for (int tile = pair; tile < P.num_tiles && ok; tile += pairs, ++n) {
        const long long t0 = (long long)(tile / P.tiles_m) * C::ROWS;
        const int m0 = (tile % P.tiles_m) * 256 + (int)rank * HALF;
        int steps = P.num_kb, nl = 0;
        for (int k = 0; k < steps; ++k, ++it) {
          const uint32_t s = it % WST, ph = (it / WST) & 1u;
          ok = stage_free(it, XST, false);
          if (!ok) break;
          const uint32_t x_s = ring + (it % XST) * (NMB * X_BYTES), w_s = ring + C::W_AT + s * W_BYTES;
          const uint32_t fb = map_to_cta(full + 8 * s, 0);
          armed |= 1u << s;
          par = (par & ~(1u << s)) | (ph << s);
          if (k < P.num_kb) {
            if (rank == 0) mbar_expect_tx(full + 8 * s, 2 * NMB * X_BYTES);
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb)
              load_pair_2d(x_s + mb * X_BYTES, &P.rows, fb, k * BK, (int)(t0 + mb * 256 + rank * HALF));
            if (k == P.num_kb - 1) {                 // now the list is needed
              nl = wait_list(n, false, ok);
              if (!ok) break;
              steps += extra_steps(nl);
            }
          } else {
            const int e = k - P.num_kb, per = P.rank > BK ? 2 : 1;
            const int first = e / per * P.cap, na = min(P.cap, nl - first), r0 = (e % per) * BK;
            // an odd number of boxes of 8 or 24 rows leaves half of a 16-deep MMA step: a box past the last adapter
            // (it reads as zero) fills it
            const int boxes = na + ((na * P.box_rows) % 16 != 0 ? 1 : 0);
            const int box_bytes = P.box_rows * 128;
            if (rank == 0) mbar_expect_tx(full + 8 * s, 2 * 2 * boxes * box_bytes);
            for (int b = 0; b < boxes; ++b) {
              const int a = b < na ? (int)list[n & 1][first + b] : P.n_adapters;
              load_pair_3d(w_s + b * box_bytes, &P.out_side, fb, m0, r0, a);
              load_pair_3d(w_s + W_BYTES / 2 + b * box_bytes, &P.out_side, fb, m0 + 64, r0, a);
            }
          }
        }
        if (adapters && ok) mbar_arrive(l_empty + 8 * (n & 1));
      }
      fill_state[0] = armed;
      fill_state[1] = par;
    }
  } else if (warp == 1) {
    // ===================== MMA issuer (leader) =====================
    // The whole warp walks the loop and one elected lane issues, with the MMAs of a step unrolled: then descriptors are
    // warp-uniform and cost an add each.  (With the loop in one lane an MMA took its thread about 200 cycles to issue,
    // more than the tensor core takes to run it: 2260 cycles a step, of which 1024 are MMA time.)
    if (rank == 0) {
      uint32_t n = 0, ws = 0, wph = 0, xs = 0;       // stages of the two rings, phase of the weights'
      bool ok = true;
      const uint64_t x_desc = make_kmajor_sw128_desc(ring), wm_desc = make_mmajor_sw128_desc(ring + C::W_AT);
      const uint64_t w_desc = GRAD ? wm_desc : make_kmajor_sw128_desc(ring + C::W_AT);
      for (int tile = pair; tile < P.num_tiles && ok; tile += pairs, ++n) {
        auto next_stage = [&] {
          if (++xs == XST) xs = 0;
          if (++ws == WST) {
            ws = 0;
            wph ^= 1u;
          }
        };
        for (int k = 0; k < P.num_kb; ++k) {
          ok = wait.all(full + 8 * ws, wph);
          if (k == 0)                                // are the accumulators moved out of the way?
            ok = ok && wait.all(t_empty, (n & 1u) ^ 1u) && wait.all(t_empty + 8, (n & 1u) ^ 1u);
          if (!ok) break;
          tc_fence_after();
          const uint64_t ad = desc_of(x_desc, xs * (NMB * X_BYTES)), bd = desc_of(w_desc, ws * W_BYTES);
          constexpr uint32_t B_STEP = GRAD ? 2048 : 32;              // 16 K values: 16 rows of 128 bytes, or 32 bytes
          if (elect_one()) {
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
              for (int q = 0; q < BK / 16; ++q)
                mma_pair(tmem + mb * 256u, desc_of(ad, mb * X_BYTES + q * 32), desc_of(bd, q * B_STEP), idesc_pair(GRAD),
                         q > 0 ? 1u : (uint32_t)k);
            commit_pair(done + 8 * ws);
          }
          __syncwarp();
          next_stage();
        }
        if (!ok) break;
        if (adapters) {
          ok = wait.all(l_full + 8 * (n & 1), (n >> 1) & 1u);
          if (!ok) break;
          const int nl = list_n[n & 1], extra = extra_steps(nl), per = P.rank > BK ? 2 : 1;
          for (int e = 0; e < extra; ++e) {
            ok = wait.all(full + 8 * ws, wph);
            if (!ok) break;
            tc_fence_after();
            const uint64_t ad = desc_of(x_desc, xs * (NMB * X_BYTES)), bd = desc_of(wm_desc, ws * W_BYTES);
            const int na = min(P.cap, nl - e / per * P.cap), r0 = (e % per) * BK;
            const int k16 = P.cap > 1 ? (na * P.box_rows + 15) / 16 : (min(BK, P.rank - r0) + 15) / 16;
            if (elect_one()) {
              for (int mb = 0; mb < NMB; ++mb)
                for (int q = 0; q < k16; ++q)
                  mma_pair(tmem + mb * 256u, desc_of(ad, mb * X_BYTES + q * 32), desc_of(bd, q * 2048), idesc_pair(true), 1u);
              commit_pair(done + 8 * ws);
            }
            __syncwarp();
            next_stage();
          }
          if (!ok) break;
        }
        if (!ok) break;
        if (elect_one()) {
          commit_pair(t_full);
          commit_pair(t_full + 8);
          if (adapters) mbar_arrive(l_empty + 8 * (n & 1));
        }
        __syncwarp();
      }
    }
  } else if (warp == 2) {
    // ===================== codes and grid =====================
    if (lane == 0 && !P.hold_loads) {
      uint32_t ct = 0, armed = 0u, par = 0u;
      bool ok = true;
      for (int tile = pair; tile < P.num_tiles && ok; tile += pairs) {
        const int m0 = (tile % P.tiles_m) * 256 + (int)rank * HALF;
        for (int kb = 0; kb < P.num_kb; ++kb, ++ct) {
          const uint32_t s = ct % CS, b = ct % CB;
          ok = wait.one(c_empty + 8 * s, (ct / CS & 1u) ^ 1u);
          if (!ok) break;
          armed |= 1u << b;
          par = (par & ~(1u << b)) | ((ct / CB & 1u) << b);
          load_codes<GRAD>(P.L, m0, kb, ring + C::C_AT + s * CODE_STAGE_BYTES, c_full + 8 * b);
        }
      }
      fill_state[2] = armed;
      fill_state[3] = par;
    }
  } else if (warp == 3) {
    // ===================== adapters of the tiles' rows =====================
    if (adapters) {
      uint32_t n = 0;
      for (int tile = pair; tile < P.num_tiles; tile += pairs, ++n) {
        const int b = (int)(n & 1);
        if (!wait.all(l_empty + 8 * b, ((n >> 1) & 1u) ^ 1u)) break;
        const long long t0 = (long long)(tile / P.tiles_m) * C::ROWS;
        int a[C::ROWS / 32];
#pragma unroll
        for (int i = 0; i < C::ROWS / 32; ++i) {
          const long long t = t0 + 32 * i + lane;
          const int v = t < P.T ? row_adapter_of(P.row_adapter, t, P.n_adapters) : -1;
          a[i] = v < 0 ? NONE : v;
          own[b][32 * i + lane] = (uint16_t)a[i];
        }
        int found = 0;
        for (int last = -1; found < C::ROWS;) {
          int m = NONE;
#pragma unroll
          for (int i = 0; i < C::ROWS / 32; ++i) m = a[i] > last ? min(m, a[i]) : m;
          m = __reduce_min_sync(0xffffffffu, m);
          if (m == NONE) break;
          last = m;
          if (lane == 0) list[b][found] = (uint16_t)m;
          ++found;
        }
        if (lane == 0) list_n[b] = found;
        __syncwarp();
        if (lane == 0) mbar_arrive(l_full + 8 * b);
      }
    }
  } else if (warp < ROLE_WARPS) {
    // ===================== finished tiles =====================
    // A lane holds a row; 32 of its columns at a time go through one of two swizzled 32 x 64-byte tiles in shared memory
    // and out by a tile store.  (Stored from registers, 16 bytes of 32 rows an instruction, a 512-column tile took 18000
    // cycles, through one 32 x 128-byte tile 10700.)
    const int q = warp & 3;
    const uint32_t t_empty_leader = map_to_cta(t_empty, 0);
    uint8_t* stage = ring_ptr + C::OUT_AT + q * OUT_BYTES + lane * 64;
    const uint32_t stage_s = ring + C::OUT_AT + q * OUT_BYTES;
    uint32_t n = 0;
    bool ok = true;
    for (int tile = pair; tile < P.num_tiles && ok; tile += pairs, ++n) {
      const int m0 = (tile % P.tiles_m) * 256;
#pragma unroll 1
      for (int mb = 0; mb < NMB; ++mb) {
        const uint32_t b = (uint32_t)mb, ph = n & 1u;
        ok = wait.all(t_full + 8 * b, ph);
        if (!ok) break;
        tc_fence_after();
        const long long t = (long long)(tile / P.tiles_m) * C::ROWS + mb * 256 + rank * HALF + q * 32;
        const uint32_t taddr = tmem + b * 256u + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
        for (int c = 0; c < 256; c += OUT_COLS) {
          const uint32_t buf = (c / OUT_COLS & 1) * OUT_BUF;
          uint32_t v[2][16];
          tc_ld16(taddr + c, v[0]);
          tc_ld16(taddr + c + 16, v[1]);
          // the tile before the last has left its staging
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          tc_ld_wait();
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t* w = &v[e >> 1][8 * (e & 1)];
            uint4 o;
            o.x = float2_to_bf16x2(__uint_as_float(w[0]), __uint_as_float(w[1]));
            o.y = float2_to_bf16x2(__uint_as_float(w[2]), __uint_as_float(w[3]));
            o.z = float2_to_bf16x2(__uint_as_float(w[4]), __uint_as_float(w[5]));
            o.w = float2_to_bf16x2(__uint_as_float(w[6]), __uint_as_float(w[7]));
            *reinterpret_cast<uint4*>(stage + buf + ((e ^ ((lane >> 1) & 3)) << 4)) = o;
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (t < P.T && m0 + c < P.M) store_2d(&P.out, stage_s + buf, m0 + c, (int)t);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(t_empty_leader + 8 * b);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  } else {
    // ===================== expanding warps =====================
    const int g = (warp - ROLE_WARPS) / GROUP_WARPS;
    const int v = threadIdx.x - 32 * ROLE_WARPS - g * 32 * GROUP_WARPS;     // 0..127 within the group
    const uint32_t full_leader = map_to_cta(full, 0);
    bool waited = false, ok = true;
    uint32_t first = 0, n = 0;                       // step counter at the tile's start
    for (int tile = pair; tile < P.num_tiles && ok; tile += pairs, ++n) {
      const int m0 = (tile % P.tiles_m) * 256 + (int)rank * HALF;
      int steps = P.num_kb, nl = -1;                 // nl: not asked for yet
      for (int k = (int)((uint32_t)(g + GROUPS - (int)(first % GROUPS)) % GROUPS);; k += GROUPS) {
        if (k >= P.num_kb && nl < 0) {
          nl = wait_list(n, true, ok);
          if (!ok) break;
          steps += extra_steps(nl);
        }
        if (k >= steps) break;
        const uint32_t it = first + k, s = it % WST;
        uint8_t* x_s = ring_ptr + (it % XST) * (NMB * X_BYTES);
        uint8_t* w_s = ring_ptr + C::W_AT + s * W_BYTES;
        if (k < P.num_kb) {
          const uint32_t ct = n * P.num_kb + k, cs = ct % CS;
          ok = wait.all(c_full + 8 * (ct % CB), (ct / CB) & 1u);
          if (!ok) break;
          const uint8_t* cst = ring_ptr + C::C_AT + cs * CODE_STAGE_BYTES;
          const CodeRun r0 = read_codes<GRAD>(P.L, cst, v, m0, k), r1 = read_codes<GRAD>(P.L, cst, v + 128, m0, k);
          __syncwarp();
          if (lane == 0) mbar_arrive(c_empty + 8 * cs);
          const Weights32 e0 = expand_unit(r0), e1 = expand_unit(r1);   // in registers, before the stage is needed
          ok = stage_free(it, WST, true);
          if (!ok) break;
          write_weights(w_s, v, e0);
          write_weights(w_s, v + 128, e1);
        } else {
          if (!waited) {
            pdl_wait();                              // h is complete from here on
            waited = true;
          }
          ok = stage_free(it, WST, true) && stage_free(it, XST, true);
          if (!ok) break;
          const int e = k - P.num_kb, per = P.rank > BK ? 2 : 1;
          const int slot0 = e / per * P.cap, na = min(P.cap, nl - slot0), r0 = (e % per) * BK;
          const long long t0 = (long long)(tile / P.tiles_m) * C::ROWS;
          for (int i = v; i < NMB * HALF * 8; i += 32 * GROUP_WARPS) {
            const int ch = i & 7, row = i >> 3;      // 8 ranks, row of this CTA
            const int mb = row / HALF, in = row % HALF, local = mb * 256 + (int)rank * HALF + in;
            const int slot = P.cap > 1 ? 8 * ch / P.rank : 0, r = P.cap > 1 ? 8 * ch - slot * P.rank : r0 + 8 * ch;
            uint4 o = make_uint4(0, 0, 0, 0);
            if (slot < na && r < P.rank && own[n & 1][local] == list[n & 1][slot0 + slot]) {
              const float4* src = reinterpret_cast<const float4*>(P.h + (t0 + local) * P.rank + r);
              const float4 a = src[0], b = src[1];
              o.x = float2_to_bf16x2(a.x, a.y);
              o.y = float2_to_bf16x2(a.z, a.w);
              o.z = float2_to_bf16x2(b.x, b.y);
              o.w = float2_to_bf16x2(b.z, b.w);
            }
            *reinterpret_cast<uint4*>(x_s + mb * X_BYTES + in * 128 + ((ch ^ (in & 7)) << 4)) = o;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor core reads what was just written
        __syncwarp();
        if (lane == 0) {
          if (rank == 0) mbar_arrive(full + 8 * s);
          else mbar_arrive_cluster(full_leader + 8 * s);
        }
      }
      first += (uint32_t)steps;
      if (adapters && ok) {
        __syncwarp();
        if (lane == 0) mbar_arrive(l_empty + 8 * (n & 1));
      }
    }
    if (!waited) pdl_wait();                         // (so that this launch ends after the one it overlaps)
  }
  tc_fence_before();
  __syncthreads();
  if (abort_s) {
    // The fills that were armed must have landed and the MMAs issued must have completed before shared and tensor memory
    // are given back.  The row fills of both CTAs are counted by the leader, which the peer waits for below, together
    // with arrivals that an aborted step may lack: then the bound of the wait (10 ms a stage) is the time they are given.
    if (threadIdx.x == 0) {
      if (rank == 0) {
        const uint32_t armed = fill_state[0], par = fill_state[1];
        for (int s = 0; s < WST; ++s)
          if (armed >> s & 1u) mbar_wait_quiet(full + 8 * s, par >> s & 1u);
      }
      const uint32_t armed = fill_state[2], par = fill_state[3];
      for (int s = 0; s < CB; ++s)
        if (armed >> s & 1u) mbar_wait_quiet(c_full + 8 * s, par >> s & 1u);
    }
    if (threadIdx.x == 32 && rank == 0) {
      commit_pair(drain_bar);
      mbar_wait_quiet(drain_bar, 0u);
    }
    if (threadIdx.x == 64) {                         // loads of this CTA that the leader never armed a barrier for
      const long long t0 = clock64();
      while (clock64() - t0 < 100000LL) {
      }
    }
    __syncthreads();
  }
  cluster_sync_all();                                // both CTAs are done with tensor memory and remote arrivals
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Pairs that the current device holds at once (a persistent kernel must not launch more); 0 on error.
template <bool GRAD>
int resident_pairs(int sms, cudaLaunchConfig_t cfg) {
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    cfg.gridDim = dim3(2 * (sms / 2));
    if (cudaOccupancyMaxActiveClusters(&n, linear_pair_kernel<GRAD>, &cfg) != cudaSuccess || n < 1) return 0;
    n = n < sms / 2 ? n : sms / 2;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

template <bool GRAD>
cudaError_t launch(PairParams& P, const bf16* x, long long ldx, const bf16* y, long long ldy, const AdapterView* ad,
                   int sms, cudaStream_t stream) {
  using C = Cfg;
  const cuuint64_t xs[2] = {(cuuint64_t)P.K, (cuuint64_t)P.T}, xst[1] = {(cuuint64_t)ldx * 2};
  const cuuint32_t xb[2] = {BK, HALF};
  if (!encode_bf16(&P.rows, x, 2, xs, xst, xb)) return cudaErrorInvalidValue;
  const cuuint64_t ys[2] = {(cuuint64_t)P.M, (cuuint64_t)P.T}, yst[1] = {(cuuint64_t)ldy * 2};
  const cuuint32_t yb[2] = {OUT_COLS, 32};
  if (!encode_bf16(&P.out, y, 2, ys, yst, yb, CU_TENSOR_MAP_SWIZZLE_64B)) return cudaErrorInvalidValue;
  P.cap = P.box_rows = 1;
  if (ad) {
    P.cap = ad->rank <= BK / 2 ? BK / ad->rank : 1;
    P.box_rows = ad->rank <= BK / 2 ? ad->rank : BK;
    const cuuint64_t as[3] = {(cuuint64_t)P.M, (cuuint64_t)ad->rank, (cuuint64_t)ad->n};
    const cuuint64_t ast[2] = {(cuuint64_t)P.M * 2, (cuuint64_t)P.M * 2 * ad->rank};
    const cuuint32_t ab[3] = {64, (cuuint32_t)P.box_rows, 1};
    if (!encode_bf16(&P.out_side, ad->out, 3, as, ast, ab)) return cudaErrorInvalidValue;
  }
  const long long tiles = (long long)P.tiles_m * ((P.T + C::ROWS - 1) / C::ROWS);
  if (tiles > 0x7fffffffLL) return cudaErrorInvalidValue;
  P.num_tiles = (int)tiles;
  const auto kernel = linear_pair_kernel<GRAD>;
  const cudaError_t e = ensure_dynamic_smem((const void*)kernel, C::SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int most = resident_pairs<GRAD>(sms, cfg);
  if (most < 1) return cudaErrorNotSupported;
  cfg.gridDim = dim3(2 * (unsigned)(tiles < most ? tiles : most));
  cfg.numAttrs = ad ? 2 : 1;                         // with adapters it may start beside the shrink launch before it
  return cudaLaunchKernelEx(&cfg, kernel, P);
}

}  // namespace

cudaError_t launch_linear_pair(bool grad, const PackedLayer& L, const AdapterView* ad, long long T,
                               const int* row_adapter, const bf16* x, long long ldx, bf16* y, long long ldy,
                               const float* h, int* status, int sms, cudaStream_t stream) {
  PairParams P = {};
  P.L = L;
  P.M = grad ? L.d_in : L.d_out;
  P.K = grad ? L.d_out : L.d_in;
  P.num_kb = (P.K + BK - 1) / BK;
  P.T = T;
  P.row_adapter = row_adapter;
  P.n_adapters = ad ? ad->n : 0;
  P.rank = ad ? ad->rank : 0;
  P.h = h;
  P.tiles_m = (P.M + 255) / 256;
  P.status = status;
  P.wait_limit = g_linear_wait_limit.load(std::memory_order_relaxed);
  P.hold_loads = g_linear_hold_loads.load(std::memory_order_relaxed);
  return grad ? launch<true>(P, x, ldx, y, ldy, ad, sms, stream) : launch<false>(P, x, ldx, y, ldy, ad, sms, stream);
}

}  // namespace admmq

extern "C" void admmq_test_pair_rings(int* groups, int* stages, int* row_stages, int* code_slots, int* code_barriers) {
  *groups = admmq::GROUPS;
  *stages = admmq::Cfg::WST;
  *row_stages = admmq::Cfg::XST;
  *code_slots = admmq::Cfg::CST;
  *code_barriers = admmq::Cfg::CBARS;
}
