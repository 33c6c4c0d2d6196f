// Attention of many rows over the 8-bit cache, on the tensor cores: prompts, and pieces of them.
//   z_j = scale q . k_j,  out = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m)
//
// A tile is 256 packed rows (token, query head of one key head), as two tracks of 128 whose products alternate on the tensor
// cores while the other's softmax runs (heads wider than 128: one track of 128 rows).  Positions come 128 (64) at a time.
// Both products take fp16 operands: queries times a power of two of their row, codes as they are, and weights
//   w_j = s_b exp(z_j - m') = 2^(z_j log2 e + log2 s_b - m')
// with the value scale s_b of the block in the exponent, so that they fit fp16 whatever the scales are; the key scale
// multiplies the finished score.  The sum of weights takes w_j / s_b in fp32.  The reference m' lies 6 below a row's maximum over
// the first positions; it is raised only after a weight has passed 2^14, which is rare, so that the accumulator is hardly ever touched
// between its products, and a row's weights need not wait for its maximum.
//   warps 0-15   softmax, two threads to a row: scores from tensor memory into registers, weights back over them (the first
//                operand of the second product), the accumulator's occasional scaling, queries in and results out
//   warps 16-19  codes: from memory into registers a tile ahead, expanded into the swizzled operand tiles.  The order of
//                positions inside a product is free, so that values, which the cache keeps as words of four tokens, need no
//                transposition: position 16 b + k of the operand is token (0 1 8 9 2 3 10 11 4 5 12 13 6 7 14 15)[k] of block b
//   warp 20      issues the products; tensor memory
//   warp 21      finds the CTA's pieces of the work, ahead of the others (22 and 23: none)
// Work is shared out in equal parts (cache_schedule.cuh), a CTA an SM.
// Bound: exponentials (16 a cycle and SM: 2048 cycles for 256 x 128) and the tensor cores (2048 as well), overlapped.  Measured, 32
// query and 8 key heads of 128: the last 2048 rows of 32768 1086 us (981 TFLOP/s, 2.5 us or some 4700 cycles a step), a prompt of 8192
// 626 us (878); heads of 64 534 us, of 192 (one track) 1623, of 256 2127.  Tensor and exponential pipes are busy 44 % of the time
// each, the schedulers 50 % (9850 warp instructions a step): what is left is the chain scores, exponents, weights, second
// product of a track.  Weights lie over their scores, so that a track's next scores wait for its own second product, and for
// what the other track has before them.  A polynomial in place of a quarter of the exponentials cost 14 %.  A CTA's first
// scores are there 11 us after its start: schedule and piece 3, queries 5, first codes and product 1.
// Registers: 88 a thread where the softmax and the codes run, 40 elsewhere; the compiler spills 76 to 178 bytes of a thread.
// Waits are bounded as in the other tensor-core kernels.  Products of a CTA run in the order of their issue; scores of the
// next positions overwrite weights on that ground.
#include "../../include/admmq_testing.h"
#include "cache_schedule.cuh"
#include "linear_tc.cuh"

namespace admmq {
namespace {

constexpr int ROWS = 128, SOFT_WARPS = 16, CODE_WARPS = 4, WARPS = 24, THREADS = 32 * WARPS, MMA_WARP = SOFT_WARPS + CODE_WARPS, PLAN_WARP = MMA_WARP + 1;
constexpr int LAUNCH_REGS = 80, SOFT_REGS = 88, CODE_REGS = 88, MMA_REGS = 40;   // of a thread
static_assert(4 * SOFT_REGS + CODE_REGS + MMA_REGS <= 6 * LAUNCH_REGS, "registers");
constexpr int STAGES = 2, SCALE_SLOTS = 4, PIECE_SLOTS = 4;
constexpr int EXTRA = 3;                             // a piece's start and end, in steps
// Weights are fp16.  The first largest of a row is 2^TOP; one above 2^LIMIT raises the reference for the steps that follow, so that
// it is 2^TOP again, and one above 2^HARD_LIMIT at once, by a whole number, so that the step's other weights are scaled exactly.
// So weights down to 2^-20 of the largest have 11 bits, and those down to 2^-31 some.  (Behind a token with 99 % of the weight, 131072 and
// a million positions of one size: the result is off by 9 and 42 % with TOP 0, by 0.2 and 1.1 % with 6.  With 8 references rise more
// often: a prompt of 8192 takes 642 us in place of 626, with 10 715.)
constexpr float TOP = 6.0f, LIMIT = 14.0f, HARD_LIMIT = 15.0f;
__device__ __forceinline__ float whole_raise(float top) { return rintf(top - TOP); }
constexpr float LN2 = 0.693147180559945309f;

template <int P>
struct Cfg {
  static constexpr int TRACKS = P <= 128 ? 2 : 1;
  static constexpr int TN = P <= 128 ? 128 : 64;     // positions of a step
  static constexpr int BLOCKS = TN / CBLOCK;
  static constexpr int Q_BYTES = ROWS * P * 2;       // a track's
  static constexpr int T_BYTES = TN * P * 2;         // expanded keys or values of a step
  static constexpr int TILES_BYTES = TRACKS * Q_BYTES + 2 * STAGES * T_BYTES;
  static constexpr int SMEM = TILES_BYTES + (P == 64 ? SOFT_WARPS * 4096 : 0) + 1024;
  // score buffers: one a track, or two of the only one
  static constexpr int S_COL = 0, O_COL = 2 * TN;
  static_assert(O_COL + TRACKS * P <= 512, "tensor memory");
  static_assert(SMEM <= (227 - 16) * 1024, "shared memory, beside what is declared in the kernel");
};

// D[128][n] fp32 = A fp16 (K-major or tensor memory) B fp16 (K-major)
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t n) {
  return (1u << 4) | ((n >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Values of a load are there after the wait: named in it, so that no use of them moves ahead.
__device__ __forceinline__ void tc_ld16_wait(uint32_t (&u)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]),
                 "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15])
               :: "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&u)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
        "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
        "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_ld32_wait(uint32_t (&u)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]),
                 "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15])
               :: "memory");
  asm volatile("" : "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]),
                    "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31]));
}
__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t (&u)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tc_ld8_wait(uint32_t (&u)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7])
               :: "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t (&u)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
               "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&u)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
      "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void more_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// A value with a tag beside it, as one access of 64 bits: the elements of a vector access have no order, so that the tag could
// be seen before its value.
__device__ __forceinline__ void post_swap(uint32_t to, uint32_t tag, float value) {
  asm volatile("st.volatile.shared.b64 [%0], %1;" ::"r"(to), "l"((uint64_t)tag << 32 | __float_as_uint(value)) : "memory");
}
// Waits, within the limit, for the word with the tag.
__device__ __forceinline__ bool poll_swap(uint32_t from, uint32_t tag, float& value, const WarpWait& wait) {
  uint64_t v;
  auto look = [&] {
    asm volatile("ld.volatile.shared.b64 %0, [%1];" : "=l"(v) : "r"(from) : "memory");
    return __all_sync(0xffffffffu, (uint32_t)(v >> 32) == tag) != 0;
  };
  bool ok = look();
  if (!ok) {
    const long long t0 = clock64();
    while (!(ok = look())) {
      const bool late = *wait.abort_flag || clock64() - t0 > wait.limit;
      if (__any_sync(0xffffffffu, late)) {
        *wait.abort_flag = 1;
        raise_status(wait.status, ST_TIMEOUT);
        break;
      }
    }
  }
  value = __uint_as_float((uint32_t)v);
  return ok;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

struct ManyArgs {
  AttendArgs a;
  long long wait_limit;
  int hold_loads;
};

// Jobs of this kernel: the plan's tiles of 256 packed rows, or their halves.
template <int P>
__device__ __forceinline__ int4 job_of(const AttendArgs& a, int tile) {
  constexpr int PER = MANY_ROWS / (Cfg<P>::TRACKS * ROWS);
  int4 job = __ldg(a.pl.big + tile / PER);
  job.y += tile % PER * ROWS;
  return job;
}
// A piece as the roles take it from shared memory.
constexpr int SKIP_BIT = 27;                         // (positions end at 2^30, a step has at most eight blocks)
struct PieceJob {
  int steps;                                         // 0: there are no more
  int pos;                                           // position of its first step
  int head, request, row0, first_row, packed;        // row0: packed row of the tile's first; packed: of the request in all
  int at;                                            // position of the request's first row
  int blocks;                                        // end of what the tile sees, in blocks; from SKIP_BIT on: how many of the first
                                                     // step's blocks lie behind its window
  int part;                                          // where its partial result goes; -1: it is whole
};

template <int P>
__global__ void __launch_bounds__(THREADS, 1) attend_many_kernel(const __grid_constant__ ManyArgs A) {
  using C = Cfg<P>;
  constexpr int TRACKS = C::TRACKS, TN = C::TN, BLOCKS = C::BLOCKS, TILE = TRACKS * ROWS;
  const AttendArgs& a = A.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Schedule<THREADS> schedule;
  // full: a step's codes are expanded; empty: its products have read them; scores complete; weights in place (and the
  // scores' buffer read); accumulator complete; queries in place; scales in place; pieces.  Waits go by parity, so a waiter
  // has to know that the phase before is over and that the one after cannot be: the scales have a barrier a slot because the
  // keys' may be a phase on before a slow warp of the softmax has looked.
  __shared__ __align__(8) uint64_t bars[4 * STAGES + SCALE_SLOTS + 2 * PIECE_SLOTS + 2 + 2 + 2 + 2 + 1];
  __shared__ float4 scales[SCALE_SLOTS][BLOCKS];     // key scale, log2 of the value scale, its reciprocal
  __shared__ PieceJob pieces[PIECE_SLOTS];
  __shared__ __align__(8) uint2 swapped[2][2][2 * ROWS];   // between the two threads of a row
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const tiles_at = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t q_at = base, k_at = q_at + TRACKS * C::Q_BYTES, v_at = k_at + STAGES * C::T_BYTES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WarpWait wait = {&abort_s, a.status, A.wait_limit};
  const uint32_t k_full = smem_u32(&bars[0]), k_empty = k_full + 8 * STAGES, v_full = k_empty + 8 * STAGES, v_empty = v_full + 8 * STAGES;
  const uint32_t s_full = v_empty + 8 * STAGES, w_full = s_full + 16, o_full = w_full + 16, q_full = o_full + 16, drain_bar = q_full + 16,
                 sc_full = drain_bar + 8, p_full = sc_full + 8 * SCALE_SLOTS, p_empty = p_full + 8 * PIECE_SLOTS;

  for (int i = threadIdx.x; i < 8 * ROWS; i += THREADS) swapped[0][0][i] = make_uint2(0u, 0u);
  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(k_full + 8 * s, CODE_WARPS);
      mbar_init(k_empty + 8 * s, 1);
      mbar_init(v_full + 8 * s, CODE_WARPS);
      mbar_init(v_empty + 8 * s, 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full + 8 * x, 1);
      mbar_init(w_full + 8 * x, 2 * ROWS / 32);
      mbar_init(o_full + 8 * x, 1);
      mbar_init(q_full + 8 * x, 2 * ROWS / 32);
    }
    mbar_init(drain_bar, 1);
    for (int s = 0; s < SCALE_SLOTS; ++s) mbar_init(sc_full + 8 * s, 1);
    for (int s = 0; s < PIECE_SLOTS; ++s) {
      mbar_init(p_full + 8 * s, 1);
      mbar_init(p_empty + 8 * s, 2 * TRACKS * ROWS / 32 + CODE_WARPS + 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_launch();
  pdl_wait();
  const int n_tiles = a.pl.n_big * (MANY_ROWS / TILE);
  const auto job = [&](int tile) { return job_of<P>(a, tile); };
  const long long total = make_schedule<THREADS, TN, TILE, EXTRA>(a, job, n_tiles, schedule) * a.c.heads;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // piece n of the CTA, by all lanes of a warp; false: a wait ran out
  const auto take = [&](uint32_t n, PieceJob& p) {
    if (!wait.all(p_full + 8 * (n % PIECE_SLOTS), n / PIECE_SLOTS & 1u)) return false;
    p = pieces[n % PIECE_SLOTS];
    __syncwarp();
    if (lane == 0) mbar_arrive(p_empty + 8 * (n % PIECE_SLOTS));
    return true;
  };

  if (warp < SOFT_WARPS) {
    more_registers<SOFT_REGS>();
    // Two threads to a row, of warps w and w + 4: each has half of a step's positions, of the query and of the result.
    const int x = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
    constexpr int CW = TN / 2;                       // positions of a thread
    if (x < TRACKS) {
      const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
      const uint32_t o_col = lanes + C::O_COL + x * P + half * (P / 2);
      const int group = a.pl.group, d = a.c.d;
      // A value of each of a row's threads to the other, as a word with the exchange's number beside it; two places in turn,
      // since the other may be one exchange ahead.  false: the wait ran out.
      uint32_t swaps = 0;
      const uint32_t swap_at = smem_u32(swapped) + (x * ROWS + r) * 8;
      auto post = [&](float mine) {
        ++swaps;
        post_swap(swap_at + ((swaps & 1u) * 2 + half) * (2 * ROWS * 8), swaps, mine);
      };
      auto answer = [&](float& other) {
        return poll_swap(swap_at + ((swaps & 1u) * 2 + (half ^ 1)) * (2 * ROWS * 8), swaps, other, wait);
      };
      auto swap = [&](float mine, float& other) {
        post(mine);
        return answer(other);
      };
      // Queries come and results go by warps, a row's 16-byte chunks in neighbouring lanes: a row a lane would touch 32 lines
      // at a time.  Half a row is QC chunks; instruction i takes rows RI i + lane / QL, QL lanes to a row.
      constexpr int QC = P / 16, QL = QC & (QC - 1) ? 4 : QC <= 8 ? QC : 8, RI = 32 / QL, QN = QC / QL;   // QN: chunks of a lane
      constexpr bool AHEAD = P <= 128;               // queries are fetched ahead (32 registers) while a result leaves
      uint4 raw[AHEAD ? QL : 1];
      // (row, head) of this lane's row of the piece as one number: -1 where it has none
      auto place_of = [&](const PieceJob& p) {
        const int pr = p.row0 + x * ROWS + r;
        return pr < p.packed ? (long long)(p.first_row + pr / group) << 32 | (uint32_t)(p.head * group + pr % group) : -1LL;
      };
      auto chunk = [&](long long place, int at) {    // chunk `at` of the row at `place`
        const bf16* src = a.q + (place >> 32) * a.q_row + (uint32_t)place * a.q_head;
        return place >= 0 && 8 * at < d ? __ldg(reinterpret_cast<const uint4*>(src) + at) : make_uint4(0, 0, 0, 0);
      };
      auto fetch_query = [&](long long place) {
        if (AHEAD) {
#pragma unroll
          for (int i = 0; i < QL; ++i)
            raw[AHEAD ? i : 0] = chunk(__shfl_sync(0xffffffffu, place, RI * i + lane / QL), half * QC + lane % QL);
        }
      };
      // The rows' queries: each times a power of two, as fp16, into the operand tile; `factor` takes a row's scores to base-2
      // exponents.
      auto place_query = [&](long long place, float& factor) {
        uint32_t tops = 0;                           // of this lane's row: magnitudes are in the order of their bits
#pragma unroll(AHEAD ? 8 : 2)
        for (int i = 0; i < QL; ++i) {
          uint32_t t = 0;
#pragma unroll
          for (int c = 0; c < QN; ++c) {
            const uint4 q = AHEAD ? raw[AHEAD ? i : 0]
                                  : chunk(__shfl_sync(0xffffffffu, place, RI * i + lane / QL), half * QC + c * QL + lane % QL);
            t = __vmaxu2(__vmaxu2(t, __vmaxu2(q.x & 0x7fff7fffu, q.y & 0x7fff7fffu)), __vmaxu2(q.z & 0x7fff7fffu, q.w & 0x7fff7fffu));
          }
#pragma unroll
          for (int o = 1; o < QL; o <<= 1) t = __vmaxu2(t, __shfl_xor_sync(0xffffffffu, t, o));
          t = __shfl_sync(0xffffffffu, t, lane % RI * QL);
          if (lane / RI == i) tops = t;
        }
        float top = __uint_as_float(min(max(tops << 16, tops & 0xffff0000u), 0x7f800000u)), other;   // (infinity for NaN)
        if (!swap(top, other)) return false;
        top = fmaxf(top, other);
        float inv;
        const float up = pow2_scale_for(top, &inv);
#pragma unroll(AHEAD ? 8 : 2)
        for (int i = 0; i < QL; ++i) {
          const int row = RI * i + lane / QL, tile_row = (warp & 3) * 32 + row;
          const float by = __shfl_sync(0xffffffffu, up, row);
#pragma unroll
          for (int c = 0; c < QN; ++c) {
            const int at = half * QC + c * QL + lane % QL;
            const uint4 q = AHEAD ? raw[AHEAD ? i : 0] : chunk(__shfl_sync(0xffffffffu, place, row), at);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = bf16x2_to_float2(w[e]);
              h[e] = pack_f16(f.x * by, f.y * by);
            }
            *reinterpret_cast<uint4*>(tiles_at + x * C::Q_BYTES + at / 8 * (ROWS * 128) + tile_row * 128 + (((at & 7) ^ (tile_row & 7)) << 4)) =
                make_uint4(h[0], h[1], h[2], h[3]);
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full + 8 * x);
        factor = top < INFINITY ? a.scale_log2 * inv : __int_as_float(0x7fc00000);
        return true;
      };

      PieceJob pc;
      bool ok = take(0, pc);
      uint32_t it = 0;                               // steps so far
      float row_scale = 0.0f;
      long long place = -1;
      if (ok && pc.steps > 0) {
        place = place_of(pc);
        fetch_query(place);
        ok = place_query(place, row_scale);
      }
      for (uint32_t n = 1; ok && pc.steps > 0; ++n) {
        // position of the row within the thread's part of the piece's first step, and what every row of the track sees: up
        // to its first row's own position, from its last row's window on
        const int shift = pc.pos + half * CW;
        int here = pc.at + (pc.row0 + x * ROWS + r) / group - shift;
        int all_to = pc.at + (pc.row0 + x * ROWS) / group - shift;
        int all_from = a.window > 0 ? pc.at + (min(pc.row0 + x * ROWS + ROWS, pc.packed) - 1) / group - a.window + 1 - shift : -0x40000000;
        const uint32_t begin = it, end = it + pc.steps;
        float ref = 0.0f, l = 0.0f, raise = 0.0f;
        bool empty = true;                           // nothing seen so far
        for (; it < end; ++it, here -= TN, all_to -= TN, all_from -= TN) {
          const int sb = TRACKS == 2 ? x : (int)(it & 1u);                         // score buffer
          ok = wait.all(sc_full + 8 * (it % SCALE_SLOTS), it / SCALE_SLOTS & 1u) &&
               wait.all(s_full + 8 * sb, TRACKS == 2 ? it & 1u : it >> 1 & 1u);
          if (!ok) break;
          tc_fence_after();
          const uint32_t s_col = lanes + C::S_COL + sb * TN + half * CW;
          const float4* sc = scales[it % SCALE_SLOTS] + half * (BLOCKS / 2);
          // exponents of 32 positions from their scores, and the largest
          auto exponents = [&](uint32_t (&u)[32], int c, float reference) {
            float2* z2 = reinterpret_cast<float2*>(u);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const float2 s = *reinterpret_cast<const float2*>(&sc[2 * c + b]);
              const float k = row_scale * s.x, o = s.y - reference;
#pragma unroll
              for (int e = 0; e < 8; ++e) z2[8 * b + e] = __ffma2_rn(z2[8 * b + e], make_float2(k, k), make_float2(o, o));
            }
            if (!(32 * c + 31 <= all_to && 32 * c >= all_from)) {
              // bits of the positions that are seen: first <= e <= last.  (A branch indeed: turned into selections it would
              // cost every step half as much again.)
              asm volatile("");
              const int last = here - 32 * c, first = a.window > 0 ? last - a.window + 1 : 0;
              const uint32_t to = last < 0 ? 0u : last >= 31 ? 0xffffffffu : (2u << last) - 1u;
              const uint32_t from = first <= 0 ? 0xffffffffu : first > 31 ? 0u : 0xffffffffu << first;
              const uint32_t seen = to & from;
#pragma unroll
              for (int e = 0; e < 32; ++e) u[e] = seen >> e & 1u ? u[e] : 0xff800000u;
            }
            const float* f = reinterpret_cast<const float*>(u);
            float tops[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) tops[i] = max3(max3(f[i], f[4 + i], f[8 + i]), max3(f[12 + i], f[16 + i], f[20 + i]), fmaxf(f[24 + i], f[28 + i]));
            return fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
          };
          auto scale_weights = [&](uint32_t col, int n, float f) {   // those of this step that are there, n columns of them
            tc_st_wait();
#pragma unroll 1
            for (int c = 0; c < n; c += 8) {
              uint32_t o[8];
              tc_ld8(col + c, o);
              tc_ld8_wait(o);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                // (in fp32: the factor itself may be below what fp16 holds, where the products are not)
                const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&o[e]));
                o[e] = pack_f16(v.x * f, v.y * f);
              }
              tc_st8(col + c, o);
            }
          };
          auto scale_accumulator = [&](float f) {    // the thread's half of it, of the products before this step
            if (!wait.all(o_full + 8 * x, (it - 1) & 1u)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < P / 2; c += 16) {
              uint32_t o[16];
              tc_ld16(o_col + c, o);
              tc_ld16_wait(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tc_st16(o_col + c, o);
            }
            return true;
          };
          if (__any_sync(0xffffffffu, raise > 0.0f)) {   // the step before asked for a higher reference
            const float f = exp2_fast(-raise);
            ok = scale_accumulator(f);
            if (!ok) break;
            ref += raise;
            l *= f;
          }
          // ---- weights, in the order of the values' operand, over the scores that they come from, 32 at a time.  `up`: how
          // far a weight that fp16 would not hold has raised the thread's reference in this step.  (Loads from tensor memory
          // that follow stores take as long as these, some 300 cycles; the first weights leave after the last load.)
          float up = 0.0f, peak = -INFINITY, add = 0.0f;
          uint32_t w[16];
#pragma unroll
          for (int c = 0; c < CW / 32; ++c) {
            uint32_t u[32];
            tc_ld32(s_col + 32 * c, u);
            tc_ld32_wait(u);
            if (c > 0) tc_st16(s_col + 16 * (c - 1), w);
            float top = exponents(u, c, ref + up);
            if (__any_sync(0xffffffffu, empty)) {      // rows that have seen nothing: their reference is the first maximum
              float other;
              ok = swap(top, other);
              if (!ok) break;
              const float most = fmaxf(top, other);
              if (empty && most > -INFINITY) {
                empty = false;
                ref = most - TOP;
                top -= ref;
#pragma unroll
                for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) - ref);
              }
            }
            peak = fmaxf(peak, top + up);
            if (__any_sync(0xffffffffu, top > HARD_LIMIT)) {
              const float by = top > HARD_LIMIT ? whole_raise(top) : 0.0f, f = exp2_fast(-by);
              scale_weights(s_col, 16 * c, f);
              add *= f;
              up += by;
#pragma unroll
              for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) - by);
            }
            float2* y = reinterpret_cast<float2*>(u);
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = make_float2(exp2_fast(y[e].x), exp2_fast(y[e].y));
#pragma unroll
            for (int b = 0; b < 2; ++b, y += 8) {
              const float2 t = __fadd2_rn(__fadd2_rn(__fadd2_rn(y[0], y[1]), __fadd2_rn(y[2], y[3])),
                                          __fadd2_rn(__fadd2_rn(y[4], y[5]), __fadd2_rn(y[6], y[7])));
              add = fmaf(t.x + t.y, sc[2 * c + b].z, add);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w[8 * b + 2 * e] = pack_f16(y[e].x, y[e].y);
                w[8 * b + 2 * e + 1] = pack_f16(y[4 + e].x, y[4 + e].y);
              }
            }
          }
          if (!ok) break;
          post(peak);                                // (read when the stores are on their way)
          tc_st16(s_col + CW / 2 - 16, w);
          float other;
          ok = answer(other);
          if (!ok) break;
          peak = fmaxf(peak, other);
          raise = peak > LIMIT ? peak - TOP : 0.0f;
          if (__any_sync(0xffffffffu, peak > HARD_LIMIT)) {   // it cannot wait for the next step
            const float by = peak > HARD_LIMIT ? whole_raise(peak) : 0.0f, f = exp2_fast(-by), f_step = exp2_fast(up - by);
            scale_weights(s_col, CW / 2, f_step);
            add *= f_step;
            if (it > begin) {
              ok = scale_accumulator(f);
              if (!ok) break;
            }
            l *= f;
            ref += by;
            raise = peak > HARD_LIMIT ? 0.0f : raise;
          }
          l += add;
          tc_st_wait();
          // One track's scores are issued ahead of the products before: the last but one has to be known to be over before
          // the last is waited for, and asked for while the last cannot be.
          if (TRACKS == 1 && it > begin && it + 1 == end) {
            ok = wait.all(o_full + 8 * x, (it - 1) & 1u);
            if (!ok) break;
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(w_full + 8 * sb);
        }
        if (!ok) break;

        // ---- result; the next piece's query is fetched meanwhile (its tile's scores are complete)
        PieceJob next;
        ok = take(n, next);
        if (!ok) break;
        const long long next_place = place_of(next);
        fetch_query(next_place);                     // (nothing where there is none: its rows are 0)
        float other;
        ok = swap(l, other) && wait.all(o_full + 8 * x, (it - 1) & 1u);
        if (!ok) break;
        l = half == 0 ? l + other : other + l;       // (one order for both)
        tc_fence_after();
        const bool complete = pc.part < 0;
        const long long slot = (long long)pc.part * TILE + x * ROWS + r;
        // by way of shared memory, 32 columns of the warp's rows at a time: where the warp puts queries (nothing reads them
        // now), or beside them where they take too little room
        const float inv = !complete ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
        uint8_t* const stage = tiles_at + (warp & 3) * 4096 + (P == 64 ? C::TILES_BYTES + (2 * x + half) * 16384 : x * C::Q_BYTES + half * (P / 64 - 1) * 16384);
#pragma unroll 1
        for (int i = 0; i < P / 2; i += 32) {
          uint32_t o[32];
          tc_ld32(o_col + i, o);
          tc_ld32_wait(o);
          const int c = half * (P / 2) + i;
          if (c >= d) continue;
          const float* f = reinterpret_cast<const float*>(o);
          __syncwarp();
          if (complete) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              *reinterpret_cast<uint4*>(stage + lane * 64 + ((k ^ (lane >> 1 & 3)) << 4)) =
                  make_uint4(float2_to_bf16x2(f[8 * k] * inv, f[8 * k + 1] * inv), float2_to_bf16x2(f[8 * k + 2] * inv, f[8 * k + 3] * inv),
                             float2_to_bf16x2(f[8 * k + 4] * inv, f[8 * k + 5] * inv), float2_to_bf16x2(f[8 * k + 6] * inv, f[8 * k + 7] * inv));
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {            // eight rows at a time, four lanes each
              const int row = 8 * k + lane / 4, col = c + 8 * (lane & 3);
              const long long at = __shfl_sync(0xffffffffu, place, row);
              const uint4 v = *reinterpret_cast<const uint4*>(stage + row * 64 + (((lane & 3) ^ (row >> 1 & 3)) << 4));
              if (at >= 0 && col < d) *reinterpret_cast<uint4*>(a.out + (at >> 32) * a.out_row + (uint32_t)at * a.out_head + col) = v;
            }
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              *reinterpret_cast<float4*>(stage + lane * 128 + ((k ^ (lane & 7)) << 4)) = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {            // four rows at a time, eight lanes each
              const int row = 4 * k + lane / 8, col = c + 4 * (lane & 7);
              const float4 v = *reinterpret_cast<const float4*>(stage + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
              if (__shfl_sync(0xffffffffu, place, row) >= 0 && col < d)
                *reinterpret_cast<float4*>(a.part + (slot - r + (warp & 3) * 32 + row) * P + col) = v;
            }
          }
        }
        tc_fence_before();
        const float top = empty ? -INFINITY : ref;
        if (place >= 0 && half == 0) {
          if (!complete) a.part_ml[slot] = make_float2(top, l);
          else if (a.lse) a.lse[(place >> 32) * (a.c.heads * group) + (uint32_t)place] = l == 0.0f ? -INFINITY : top * LN2 + logf(l);
        }
        place = next_place;
        __syncwarp();                                // (the staged rows are read before queries go over them)
        if (next.steps > 0) ok = place_query(place, row_scale);
        pc = next;
      }
    }
  } else if (warp < MMA_WARP) {
    more_registers<CODE_REGS>();
    const int w = warp - SOFT_WARPS, tid = threadIdx.x - 32 * SOFT_WARPS;
    // Three steps are under way: one is expanded, the codes of the next are on their way, and the pages of the one after
    // are looked up.  Lanes 0 .. BLOCKS - 1 hold a block each.
    struct Look {                                    // a step whose pages have been asked for
      int page, block, heads_before;                 // page -1: none;  block of the page;  head * blocks of a page
      bool more;                                     // is there such a step?
    };
    struct Found {                                   // a step whose codes can be asked for
      int at;                                        // block of the cache, -1: none (block 0 is read for it, unused)
      float2 scale;
      bool more;
    };
    PieceJob pc;
    uint32_t n_piece = 0;
    int left = 0;
    bool ended = false;                              // no more pieces, or a wait ran out
    auto look = [&]() {
      Look n = {-1, 0, 0, false};
      int skip = 0;
      if (left == 0) {
        ended = ended || !take(n_piece++, pc) || pc.steps == 0;
        if (ended) return n;
        left = pc.steps;
        skip = pc.blocks >> SKIP_BIT;                // (blocks behind the window are not asked for: their pages may be gone)
        pc.blocks &= (1 << SKIP_BIT) - 1;
      }
      n.more = true;
      const int b = pc.pos / CBLOCK + lane;
      if (lane < BLOCKS && lane >= skip && b < pc.blocks) {
        n.page = a.pl.tables[(long long)pc.request * a.pl.max_pages + (b >> a.c.bpp_shift)];
        n.block = b & a.c.bpp - 1;
        if (n.page < 0) n.page = 0x7fffffff;         // (-1 is "none", not a page that does not exist)
      }
      n.heads_before = pc.head * a.c.bpp;
      --left;
      pc.pos += TN;
      return n;
    };
    auto find = [&](const Look& n) {
      Found f = {-1, make_float2(0.f, 0.f), n.more};
      if (n.page >= a.c.n_pages) raise_status(a.status, ADMMQ_ERR_SHAPE);
      else if (n.page >= 0) {
        f.at = n.page * (a.c.heads * a.c.bpp) + n.heads_before + n.block;
        f.scale = __ldg(a.c.scale + f.at);
      }
      return f;
    };
    // Keys: chunk (h, i) of this thread is quarter kq of the 64 values from 64 h on of token kt + 32 i.  Values: chunk e is
    // what lane (vg, 2 vu) and its neighbour hold (32 bytes) of a block and 32 columns; a warp takes two blocks.
    constexpr int KH = P / 64, KI = TN / 32, PAIRS = BLOCKS / 2, VE = P / 32 * PAIRS / CODE_WARPS;
    uint4 kr[KH][KI], vr[VE][2];
    const int kq = tid & 3, kt = tid >> 2;
    const int vu = lane & 1, vb = lane >> 1 & 1, vg = (lane >> 2 & 1) | (lane >> 3) << 1;
    const int vblk = 2 * (w % PAIRS) + vb, vc = w / PAIRS;            // (columns 32 (vc + CODE_WARPS / PAIRS e))
    const uint32_t k_src = kt % CBLOCK * 64 + kq * 16, v_src = 16 * P + vc * 512 + vg * 64 + vu * 32;
    const uint32_t k_dst = kt * 128 + ((2 * kq) ^ (kt & 7)) * 16;      // (the neighbouring chunk: address ^ 16)
    const uint32_t v_dst = vblk / 4 * (P * 128) + (32 * vc + 4 * vg) * 128;
    auto fetch_k = [&](int at) {
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int b = max(0, __shfl_sync(0xffffffffu, at, kt / CBLOCK + 2 * i));
        const uint8_t* src = a.c.codes + (size_t)(uint32_t)b * (uint32_t)(32 * P) + k_src;
#pragma unroll
        for (int h = 0; h < KH; ++h) kr[h][i] = ldg_stream(src + h * 1024);
      }
    };
    auto fetch_v = [&](int at) {
      const int b = max(0, __shfl_sync(0xffffffffu, at, vblk));
      const uint8_t* src = a.c.codes + (size_t)(uint32_t)b * (uint32_t)(32 * P) + v_src;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        vr[e][0] = ldg_stream(src + e * (CODE_WARPS / PAIRS * 512));
        vr[e][1] = ldg_stream(src + e * (CODE_WARPS / PAIRS * 512) + 16);
      }
    };
    if (!A.hold_loads) {
      Found now = find(look()), next;
      fetch_k(now.at);
      fetch_v(now.at);
      Look ahead = look();
      for (uint32_t it = 0; now.more; ++it) {
        const uint32_t s = it % STAGES, ph = it / STAGES & 1u;
        next = find(ahead);
        ahead = look();
        if (!wait.all(k_empty + 8 * s, ph ^ 1u)) break;
        uint8_t* const to_k = tiles_at + TRACKS * C::Q_BYTES + s * C::T_BYTES;
#pragma unroll
        for (int h = 0; h < KH; ++h)
#pragma unroll
          for (int i = 0; i < KI; ++i) {
            const uint4 c = kr[h][i];
            uint8_t* dst = to_k + h * (TN * 128) + i * 4096;
            *reinterpret_cast<uint4*>(dst + k_dst) =
                make_uint4(two_codes<false>(c.x), two_codes<true>(c.x), two_codes<false>(c.y), two_codes<true>(c.y));
            *reinterpret_cast<uint4*>(dst + (k_dst ^ 16)) =
                make_uint4(two_codes<false>(c.z), two_codes<true>(c.z), two_codes<false>(c.w), two_codes<true>(c.w));
          }
        if (w == 0 && lane < BLOCKS) {
          const ValueScale vs = value_scale(now.scale.y);
          scales[it % SCALE_SLOTS][lane] = now.at >= 0 ? make_float4(now.scale.x, vs.log2, vs.inv, 0.f) : make_float4(0.f, -INFINITY, 0.f, 0.f);
        }
        fence_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(k_full + 8 * s);
          if (w == 0) mbar_arrive(sc_full + 8 * (it % SCALE_SLOTS));
        }
        fetch_k(next.at);
        if (!wait.all(v_empty + 8 * s, ph ^ 1u)) break;
        uint8_t* const to_v = tiles_at + TRACKS * C::Q_BYTES + (STAGES + s) * C::T_BYTES;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const uint32_t lo[4] = {vr[e][0].x, vr[e][0].y, vr[e][0].z, vr[e][0].w}, hi[4] = {vr[e][1].x, vr[e][1].y, vr[e][1].z, vr[e][1].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint4*>(to_v + e * (CODE_WARPS / PAIRS * 4096) + v_dst + k * 128 +
                                      (((2 * (vblk & 3) + vu) ^ ((4 * vg + k) & 7)) << 4)) =
                make_uint4(two_codes<false>(lo[k]), two_codes<true>(lo[k]), two_codes<false>(hi[k]), two_codes<true>(hi[k]));
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_full + 8 * s);
        fetch_v(next.at);
        now = next;
      }
    }
  } else {
    fewer_registers<MMA_REGS>();
    if (warp == MMA_WARP) {
      uint32_t it = 0;
      bool ok = true;
      // scores of step i (of the CTA's) of track x
      auto scores = [&](uint32_t i, int x) {
        const uint64_t qd = make_kmajor_sw128_desc(q_at + x * C::Q_BYTES), kd = make_kmajor_sw128_desc(k_at + i % STAGES * C::T_BYTES);
        const int sb = TRACKS == 2 ? x : (int)(i & 1u);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < P / 16; ++k)
            tc_mma_f16(tmem + C::S_COL + sb * TN, desc_of(qd, k / 4 * (ROWS * 128) + k % 4 * 32), desc_of(kd, k / 4 * (TN * 128) + k % 4 * 32),
                       idesc_f16(TN), k > 0);
          tc_commit(s_full + 8 * sb);
          if (x == TRACKS - 1) tc_commit(k_empty + 8 * (i % STAGES));
        }
        __syncwarp();
      };
      PieceJob pc;
      for (uint32_t n = 0; ok; ++n) {
        ok = take(n, pc);
        if (!ok || pc.steps == 0) break;
        const int steps = pc.steps;
        ok = wait.all(k_full + 8 * (it % STAGES), it / STAGES & 1u);
        for (int x = 0; x < TRACKS && ok; ++x) {
          ok = wait.all(q_full + 8 * x, n & 1u);
          if (!ok) break;
          tc_fence_after();
          scores(it, x);
        }
        for (int j = 0; ok && j < steps; ++j, ++it) {
          const uint32_t s = it % STAGES;
          if (TRACKS == 1 && j + 1 < steps) {        // the next scores go to the other buffer, ahead of these weights
            ok = wait.all(k_full + 8 * ((it + 1) % STAGES), (it + 1) / STAGES & 1u);
            if (!ok) break;
            tc_fence_after();
            scores(it + 1, 0);
          }
          for (int x = 0; x < TRACKS; ++x) {
            const int sb = TRACKS == 2 ? x : (int)(it & 1u);
            // (what is there long before the weights is waited for before them)
            if (x == 0) {
              ok = wait.all(v_full + 8 * s, it / STAGES & 1u);
              if (ok && TRACKS == 2 && j + 1 < steps) ok = wait.all(k_full + 8 * ((it + 1) % STAGES), (it + 1) / STAGES & 1u);
            }
            ok = ok && wait.all(w_full + 8 * sb, TRACKS == 2 ? it & 1u : it >> 1 & 1u);
            if (!ok) break;
            tc_fence_after();
            const uint64_t vd = make_kmajor_sw128_desc(v_at + s * C::T_BYTES);
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < TN / 16; ++k)
                tc_mma_f16_ts(tmem + C::O_COL + x * P, tmem + C::S_COL + sb * TN + k / (TN / 32) * (TN / 2) + k % (TN / 32) * 8, desc_of(vd, k / 4 * (P * 128) + k % 4 * 32),
                              idesc_f16(P), j > 0 || k > 0);
              tc_commit(o_full + 8 * x);
              if (x == TRACKS - 1) tc_commit(v_empty + 8 * s);
            }
            __syncwarp();
            if (TRACKS == 2 && j + 1 < steps) {
              scores(it + 1, x);
            }
          }
        }
      }
    } else if (warp == PLAN_WARP) {
      const int ctas = active_ctas(total, 1), cta = blockIdx.x;
      long long u = cta < ctas ? line_at(total, cta, ctas) : 0;
      const long long line_end = cta < ctas ? line_at(total, cta + 1, ctas) : 0;
      bool told = false;                             // of a (tile, head) that others end
      // Once a wait has run out nobody takes pieces any more; the line is walked to its end all the same, since the join
      // that follows goes by what is told of every (tile, head).
      bool heard = true;
      Piece f;
      for (uint32_t n = 0;; ++n) {
        PieceJob p = {};
        if (u < line_end) {
          // searched for once, then one after the other
          if (n == 0) {
            f = find_piece<THREADS, TN, TILE, EXTRA>(a, job, n_tiles, schedule, u);
          } else if (f.head + 1 < a.c.heads) {
            const long long cost = f.end - f.begin + EXTRA;
            ++f.head;
            f.begin += cost;
            f.end += cost;
          } else {
            int units = 0;                           // (there is a tile with some: the line goes on)
            while (units == 0 && f.tile + 1 < n_tiles) {
              f.job = job(++f.tile);
              f.span = span_of(a, f.job, TILE);
              units = units_of<TN>(f.span, f.job, a.pl.group);
            }
            f.head = 0;
            f.begin = f.end + EXTRA;
            f.end = f.begin + units;
          }
          const long long stop = min(line_end, f.end);
          u = max(u, f.begin);
          if (u < stop) {
            p.steps = (int)(stop - u);
            p.pos = ((int)(u - f.begin) + f.span.lo / TN) * TN;
            p.head = f.head;
            p.request = f.job.x;
            p.row0 = f.job.y;
            p.first_row = f.job.z;
            p.packed = f.job.w * a.pl.group;
            p.at = f.span.at;
            p.blocks = (f.span.hi + CBLOCK - 1) / CBLOCK | max(0, f.span.lo / CBLOCK - p.pos / CBLOCK) << SKIP_BIT;
            p.part = u == f.begin && stop == f.end ? -1 : 2 * cta + (u == f.begin ? 1 : 0);
            if (u == f.begin) {
              told = stop < f.end;
              if (lane == 0) tell_join(a, f, TILE, cta, told ? cta_of(f.end - 1, total, ctas) : cta);
            }
            u = stop;
          }
        }
        heard = heard && wait.all(p_empty + 8 * (n % PIECE_SLOTS), (n / PIECE_SLOTS & 1u) ^ 1u);
        if (heard && lane == 0) {
          pieces[n % PIECE_SLOTS] = p;
          mbar_arrive(p_full + 8 * (n % PIECE_SLOTS));
        }
        __syncwarp();
        if (p.steps == 0) break;
        if (!heard) continue;
        // its queries into the L2 cache: fetched when the piece before ends, they would keep the softmax waiting for memory
        for (int i = lane; n > 0 && i < TILE && p.row0 + i < p.packed; i += 32) {
          const int pr = p.row0 + i, g = a.pl.group;
          const bf16* src = a.q + (long long)(p.first_row + pr / g) * a.q_row + (p.head * g + pr % g) * a.q_head;
          for (int c = 0; c < a.c.d; c += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + c));
        }
      }
      if (lane == 0 && !told) tell_none(a, cta);
    }
  }
  __syncthreads();
  if (abort_s && threadIdx.x == 32 * MMA_WARP) {     // (no copies to wait for; products in flight still use their operands)
    tc_commit(drain_bar);
    mbar_wait_quiet(drain_bar, 0u);
  }
  __syncthreads();
  if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

bool has_registers(const void* kernel) {
  cudaFuncAttributes attr;
  return cudaFuncGetAttributes(&attr, kernel) == cudaSuccess && attr.numRegs == LAUNCH_REGS;
}

template <int P>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t stream) {
  using C = Cfg<P>;
  const cudaError_t e = ensure_dynamic_smem((const void*)attend_many_kernel<P>, C::SMEM);
  if (e != cudaSuccess) return e;
  // (with fewer registers at launch the warps would wait for more than there are)
  static const bool registers = has_registers((const void*)attend_many_kernel<P>);
  if (!registers) return cudaErrorInvalidConfiguration;
  const ManyArgs args = {a, g_linear_wait_limit.load(std::memory_order_relaxed), g_linear_hold_loads.load(std::memory_order_relaxed)};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sms);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, attend_many_kernel<P>, args);
}

}  // namespace

cudaError_t launch_cache_attend_many(const AttendArgs& a, cudaStream_t stream) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  cudaError_t e;
  switch (a.c.p / 64) {
    case 1: e = launch<64>(a, sms, stream); break;
    case 2: e = launch<128>(a, sms, stream); break;
    case 3: e = launch<192>(a, sms, stream); break;
    default: e = launch<256>(a, sms, stream); break;
  }
  return e == cudaSuccess ? launch_cache_join(a, true, sms, stream) : e;
}

}  // namespace admmq
