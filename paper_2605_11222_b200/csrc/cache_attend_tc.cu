// Attention of many rows over the 8-bit cache, on the tensor cores: prompts, and pieces of them.
//   z_j = scale q . k_j,  out = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m)
//
// A tile is 256 packed rows (token, query head of one key head), as two tracks of 128 whose products alternate on the tensor
// cores while the other's softmax runs (heads wider than 128: one track of 128 rows).  Positions come 128 (64) at a time.
// Both products take fp16 operands: queries times a power of two of their row, codes as they are, and weights
//   w_j = s_b exp(z_j - m') = 2^(z_j log2 e + log2 s_b - m')
// with the value scale s_b of the block in the exponent, so that they stay below 2^8 whatever the scales are; the key scale
// multiplies the finished score.  The sum of weights takes w_j / s_b.  The accumulators' reference m' is raised only when a
// weight would pass 2^8, which is rare, so that the accumulator is hardly ever touched between its products.
//   warps 0-7    softmax, a row a thread: scores from tensor memory into registers, weights back over them (the first
//                operand of the second product), the accumulator's occasional scaling, queries in and results out
//   warps 8-11   codes: from memory into registers a tile ahead, expanded into the swizzled operand tiles.  The order of
//                positions inside a product is free, so that values, which the cache keeps as words of four tokens, need no
//                transposition: position 16 b + k of the operand is token (0 1 8 9 2 3 10 11 4 5 12 13 6 7 14 15)[k] of block b
//   warp 12      issues the products; tensor memory
// Work is shared out in equal parts (cache_schedule.cuh), a CTA an SM.
// Bound: exponentials (16 a cycle and SM: 2048 cycles for 256 x 128) and the tensor cores (2048 as well), overlapped.
// Waits are bounded as in the other tensor-core kernels.  Products of a CTA run in the order of their issue; scores of the
// next positions overwrite weights on that ground.
#include "../../include/admmq_testing.h"
#include "cache_schedule.cuh"
#include "linear_tc.cuh"

namespace admmq {
namespace {

constexpr int ROWS = 128, SOFT_WARPS = 8, CODE_WARPS = 4, WARPS = 16, THREADS = 32 * WARPS, MMA_WARP = SOFT_WARPS + CODE_WARPS;
constexpr int SOFT_REGS = 184, CODE_REGS = 104, MMA_REGS = 40;     // of 128 each at launch
static_assert(2 * SOFT_REGS + CODE_REGS + MMA_REGS <= 4 * 128, "registers");
constexpr int STAGES = 2, SCALE_SLOTS = 4;
constexpr int EXTRA = 3;                             // a piece's start and end, in steps
constexpr float LIMIT = 8.0f;                        // weights stay below 2^LIMIT
constexpr float LN2 = 0.693147180559945309f;

template <int P>
struct Cfg {
  static constexpr int TRACKS = P <= 128 ? 2 : 1;
  static constexpr int TN = P <= 128 ? 128 : 64;     // positions of a step
  static constexpr int BLOCKS = TN / CBLOCK;
  static constexpr int Q_BYTES = ROWS * P * 2;       // a track's
  static constexpr int T_BYTES = TN * P * 2;         // expanded keys or values of a step
  static constexpr int SMEM = TRACKS * Q_BYTES + 2 * STAGES * T_BYTES + 1024;
  // score buffers: one a track, or two of the only one
  static constexpr int S_COL = 0, O_COL = 2 * TN;
  static_assert(O_COL + TRACKS * P <= 512, "tensor memory");
  static_assert(SMEM <= 227 * 1024 - 8192, "shared memory");
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
__device__ __forceinline__ void tc_ld32(uint32_t taddr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
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
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
      ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
      "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]),
      "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]),
      "r"(u[31]), "r"(taddr)
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

// Bounded wait of a whole warp with one answer for all its lanes.  (Inlined: setmaxnreg asks for a kernel without calls.)
struct WarpWait {
  volatile int* abort_flag;
  int* status;
  long long limit;
  __device__ __forceinline__ bool all(uint32_t bar, uint32_t parity) const {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status, limit)) != 0;
  }
};

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

template <int P>
__global__ void __launch_bounds__(THREADS, 1) attend_many_kernel(const __grid_constant__ ManyArgs A) {
  using C = Cfg<P>;
  constexpr int TRACKS = C::TRACKS, TN = C::TN, BLOCKS = C::BLOCKS, TILE = TRACKS * ROWS;
  const AttendArgs& a = A.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Schedule<THREADS> schedule;
  // full: a step's codes are expanded; empty: its products have read them; scores complete; weights in place (and the
  // scores' buffer read); accumulator complete; queries in place; scales in place.  Waits go by parity, so a waiter has to
  // know that the phase before is over and that the one after cannot be: the scales have a barrier a slot because the keys'
  // may be a phase on before a slow warp of the softmax has looked.
  __shared__ __align__(8) uint64_t bars[4 * STAGES + SCALE_SLOTS + 2 + 2 + 2 + 2 + 1];
  __shared__ float4 scales[SCALE_SLOTS][BLOCKS];     // key scale, log2 of the value scale, its reciprocal
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const tiles_at = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t q_at = base, k_at = q_at + TRACKS * C::Q_BYTES, v_at = k_at + STAGES * C::T_BYTES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WarpWait wait = {&abort_s, a.status, A.wait_limit};
  const uint32_t k_full = smem_u32(&bars[0]), k_empty = k_full + 8 * STAGES, v_full = k_empty + 8 * STAGES, v_empty = v_full + 8 * STAGES;
  const uint32_t s_full = v_empty + 8 * STAGES, w_full = s_full + 16, o_full = w_full + 16, q_full = o_full + 16, drain_bar = q_full + 16,
                 sc_full = drain_bar + 8;

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
      mbar_init(w_full + 8 * x, ROWS / 32);
      mbar_init(o_full + 8 * x, 1);
      mbar_init(q_full + 8 * x, ROWS / 32);
    }
    mbar_init(drain_bar, 1);
    for (int s = 0; s < SCALE_SLOTS; ++s) mbar_init(sc_full + 8 * s, 1);
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
  const int ctas = active_ctas(total, 1), cta = blockIdx.x;
  const long long line_begin = cta < ctas ? line_at(total, cta, ctas) : 0, line_end = cta < ctas ? line_at(total, cta + 1, ctas) : 0;
  const auto piece = [&](long long u) { return find_piece<THREADS, TN, TILE, EXTRA>(a, job, n_tiles, schedule, u); };

  if (warp < SOFT_WARPS) {
    more_registers<SOFT_REGS>();
    const int x = warp >> 2, r = (warp & 3) * 32 + lane;
    if (x < TRACKS) {
      const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
      const uint32_t o_col = lanes + C::O_COL + x * P;
      const int group = a.pl.group, d = a.c.d;
      int4 join = make_int4(-1, 0, 0, 0);
      uint32_t it = 0, n_piece = 0;                  // steps and pieces so far
      bool ok = true;
      for (long long u = line_begin; ok && u < line_end; ++n_piece) {
        const Piece pc = piece(u);
        const long long stop = min(line_end, pc.end);
        u = max(u, pc.begin);
        if (u >= stop) break;
        const int steps = (int)(stop - u), pr = pc.job.y + x * ROWS + r, packed = pc.job.w * group;
        if (u == pc.begin && stop < pc.end) join = make_int4(pc.tile, pc.head, cta_of(pc.end - 1, total, ctas), 0);
        const int token = pr / group, head = pc.head * group + pr % group;
        const bool mine = pr < packed;

        // ---- the row's query: times a power of two, as fp16
        float row_scale;
        {
          const bf16* src = a.q + (long long)(pc.job.z + token) * a.q_row + head * a.q_head;
          float top = 0.0f;
          bool finite = true;
          auto chunk = [&](int c) { return mine && 8 * c < d ? __ldg(reinterpret_cast<const uint4*>(src) + c) : make_uint4(0, 0, 0, 0); };
#pragma unroll 8
          for (int c = 0; c < P / 8; ++c) {
            const uint4 q = chunk(c);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = bf16x2_to_float2(w[e]);
              top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
              finite &= isfinite(f.x) && isfinite(f.y);
            }
          }
          float inv;
          const float up = pow2_scale_for(top, &inv);
          row_scale = finite ? a.scale_log2 * inv : __int_as_float(0x7fc00000);
          uint8_t* dst = tiles_at + x * C::Q_BYTES + r * 128;
#pragma unroll 8
          for (int c = 0; c < P / 8; ++c) {
            const uint4 q = chunk(c);                // (from the L1 cache)
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = bf16x2_to_float2(w[e]);
              h[e] = pack_f16(f.x * up, f.y * up);
            }
            *reinterpret_cast<uint4*>(dst + c / 8 * (ROWS * 128) + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(q_full + 8 * x);
        }

        const int here = pc.span.at + token;
        // positions that every row of the track sees: up to its first row's own, from its last row's window on
        const int track_first = pc.job.y + x * ROWS;
        const int all_to = pc.span.at + track_first / group;
        const int all_from = a.window > 0 ? pc.span.at + (min(track_first + ROWS, packed) - 1) / group - a.window + 1 : 0;
        int pos = ((int)(u - pc.begin) + pc.span.lo / TN) * TN;
        float ref = 0.0f, l = 0.0f;
        bool empty = true;                           // nothing seen so far
        for (int j = 0; j < steps; ++j, ++it, pos += TN) {
          const int sb = TRACKS == 2 ? x : (int)(it & 1u);                         // score buffer
          const uint32_t phase = TRACKS == 2 ? it & 1u : it >> 1 & 1u;
          ok = wait.all(sc_full + 8 * (it % SCALE_SLOTS), it / SCALE_SLOTS & 1u) && wait.all(s_full + 8 * sb, phase);
          if (!ok) break;
          tc_fence_after();
          float z[TN];
          const uint32_t s_col = lanes + C::S_COL + sb * TN;
#pragma unroll
          for (int c = 0; c < TN / 32; ++c) tc_ld32(s_col + 32 * c, z + 32 * c);
          tc_ld_wait();
          const float4* sc = scales[it % SCALE_SLOTS];
          float2* z2 = reinterpret_cast<float2*>(z);
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            const float4 s = sc[b];
            const float k = row_scale * s.x, c = s.y - ref;
#pragma unroll
            for (int e = 0; e < 8; ++e) z2[8 * b + e] = __ffma2_rn(z2[8 * b + e], make_float2(k, k), make_float2(c, c));
          }
          const bool whole = pos + TN - 1 <= all_to && pos >= all_from;
          if (!whole) {
            const int last = here - pos, first = a.window > 0 ? here - a.window + 1 - pos : 0;
#pragma unroll
            for (int e = 0; e < TN; ++e)
              if (e > last || e < first) z[e] = -INFINITY;
          }
          float most = z[0];
#pragma unroll
          for (int e = 1; e < TN; ++e) most = fmaxf(most, z[e]);
          const bool raise = empty ? most > -INFINITY : most > LIMIT;
          if (__any_sync(0xffffffffu, raise)) {
            const float by = raise ? most : 0.0f, f = raise ? (empty ? 0.0f : exp2_fast(-most)) : 1.0f;
            ref += by;
            l *= f;
#pragma unroll
            for (int e = 0; e < TN / 2; ++e) z2[e] = __fadd2_rn(z2[e], make_float2(-by, -by));
            empty = empty && !raise;
            if (j > 0) {
              ok = wait.all(o_full + 8 * x, (it - 1) & 1u);
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < P; c += 32) {
                float o[32];
                tc_ld32(o_col + c, o);
                tc_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] *= f;
                tc_st32(o_col + c, reinterpret_cast<const uint32_t*>(o));
              }
            }
          }
          // ---- weights, in the order of the values' operand
#pragma unroll
          for (int c = 0; c < TN / 64; ++c) {
            uint32_t w[32];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              float* y = z + 64 * c + 16 * b;
              const float2* y2 = reinterpret_cast<const float2*>(y);
#pragma unroll
              for (int e = 0; e < 16; ++e) y[e] = exp2_fast(y[e]);
              float2 s = make_float2(0.f, 0.f);
#pragma unroll
              for (int e = 0; e < 8; ++e) s = __fadd2_rn(s, y2[e]);
              const float sum = s.x + s.y;
              // (a block that the row sees nothing of adds nothing, even with a scale of NaN)
              l = sum == 0.0f ? l : fmaf(sum, sc[4 * c + b].z, l);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w[8 * b + 2 * e] = pack_f16(y2[e].x, y2[e].y);
                w[8 * b + 2 * e + 1] = pack_f16(y2[4 + e].x, y2[4 + e].y);
              }
            }
            tc_st32(s_col + 32 * c, w);
          }
          tc_st_wait();
          // One track's scores are issued ahead of the products before: the last but one has to be known to be over before
          // the last is waited for, and asked for while the last cannot be.
          if (TRACKS == 1 && j > 0 && j == steps - 1) {
            ok = wait.all(o_full + 8 * x, (it - 1) & 1u);
            if (!ok) break;
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(w_full + 8 * sb);
        }
        if (!ok) break;

        // ---- result
        ok = wait.all(o_full + 8 * x, (it - 1) & 1u);
        if (!ok) break;
        tc_fence_after();
        const bool complete = u == pc.begin && stop == pc.end;
        const float inv = !complete ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
        const long long row = pc.job.z + token;
        const int slot = (2 * cta + (u == pc.begin ? 1 : 0)) * TILE + x * ROWS + r;
#pragma unroll 1
        for (int c = 0; c < P; c += 32) {
          float o[32];
          tc_ld32(o_col + c, o);
          tc_ld_wait();
          if (mine) {
            if (complete) {
              uint4* dst = reinterpret_cast<uint4*>(a.out + row * a.out_row + head * a.out_head + c);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (c + 8 * i < d)
                  dst[i] = make_uint4(float2_to_bf16x2(o[8 * i] * inv, o[8 * i + 1] * inv), float2_to_bf16x2(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                                      float2_to_bf16x2(o[8 * i + 4] * inv, o[8 * i + 5] * inv), float2_to_bf16x2(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
            } else {
              float4* dst = reinterpret_cast<float4*>(a.part + (long long)slot * P + c);
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (c + 4 * i < d) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          }
        }
        tc_fence_before();
        const float top = empty ? -INFINITY : ref;
        if (mine) {
          if (!complete) a.part_ml[slot] = make_float2(top, l);
          else if (a.lse) a.lse[row * (a.c.heads * group) + head] = l == 0.0f ? -INFINITY : top * LN2 + logf(l);
        }
        u = stop;
      }
      if (threadIdx.x == 0) a.joins[cta] = join;
    }
  } else if (warp < MMA_WARP) {
    fewer_registers<CODE_REGS>();
    const int w = warp - SOFT_WARPS, tid = threadIdx.x - 32 * SOFT_WARPS;
    constexpr int K_EACH = TN * P / 16 / (32 * CODE_WARPS), V_EACH = K_EACH / 2;   // 16-byte chunks of keys, 32 of values
    // the step that is fetched next
    long long u = line_begin;
    Piece pc;
    int left = 0, blk0 = 0;
    auto places = [&](float4* scale, bool& more) -> long long {  // byte offset of the lane's block (lanes 0 .. BLOCKS - 1), -1: none
      more = false;
      if (left == 0) {
        if (u >= line_end) return -1;
        pc = piece(u);
        const long long stop = min(line_end, pc.end);
        u = max(u, pc.begin);
        if (u >= stop) return -1;
        left = (int)(stop - u);
        blk0 = ((int)(u - pc.begin) + pc.span.lo / TN) * BLOCKS;
        u = stop;
      }
      more = true;
      long long at = -1;
      *scale = make_float4(0.f, -INFINITY, 0.f, 0.f);
      const int b = blk0 + lane;
      if (lane < BLOCKS && b < (pc.span.hi + CBLOCK - 1) / CBLOCK) {
        at = block_index(a.c, a.pl, pc.job.x, b, a.status);
        if (at >= 0) {
          at += (long long)pc.head * a.c.bpp;
          const float2 s = __ldg(a.c.scale + at);
          const float vs = s.y == 0.0f ? 1.0f : s.y;
          *scale = make_float4(s.x, __log2f(vs), __fdividef(1.0f, vs), 0.f);
          at *= a.c.block_bytes;
        }
      }
      --left;
      blk0 += BLOCKS;
      return at;
    };
    uint4 kr[K_EACH], vr[2 * V_EACH];
    // key chunk e of this thread: token, quarter of a 64-value column, column
    auto fetch_k = [&](long long place) {
#pragma unroll
      for (int e = 0; e < K_EACH; ++e) {
        const int i = e * 32 * CODE_WARPS + tid, token = i / 4 % TN, h = i / (4 * TN);
        const long long at = __shfl_sync(0xffffffffu, place, token / CBLOCK);
        kr[e] = at >= 0 ? ldg_stream(a.c.codes + at + h * 1024 + token % CBLOCK * 64 + (i & 3) * 16) : make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
      }
    };
    // value chunk e: two blocks by lane, g, and pairs of t; 32-value column
    const int vu = lane & 1, vb = lane >> 1 & 1, vg = (lane >> 2 & 1) | (lane >> 3) << 1;
    auto fetch_v = [&](long long place) {
#pragma unroll
      for (int e = 0; e < V_EACH; ++e) {
        const int i = e * CODE_WARPS + w, pair = i % (BLOCKS / 2), c = i / (BLOCKS / 2);
        const long long at = __shfl_sync(0xffffffffu, place, 2 * pair + vb);
        const uint8_t* p = a.c.codes + at + 16 * P + c * 512 + vg * 64 + vu * 32;
        const uint4 none = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
        vr[2 * e] = at >= 0 ? ldg_stream(p) : none;
        vr[2 * e + 1] = at >= 0 ? ldg_stream(p + 16) : none;
      }
    };
    float4 scale, next_scale;
    bool more, next_more;                            // is there a step?
    if (!A.hold_loads) {
      long long place = places(&scale, more);
      fetch_k(place);
      fetch_v(place);
      for (uint32_t it = 0; more; ++it, more = next_more) {
        const uint32_t s = it % STAGES, ph = it / STAGES & 1u;
        place = places(&next_scale, next_more);
        if (!wait.all(k_empty + 8 * s, ph ^ 1u)) break;
        uint8_t* kt = tiles_at + TRACKS * C::Q_BYTES + s * C::T_BYTES;
#pragma unroll
        for (int e = 0; e < K_EACH; ++e) {
          const int i = e * 32 * CODE_WARPS + tid, token = i / 4 % TN, h = i / (4 * TN), q = i & 3;
          uint8_t* dst = kt + h * (TN * 128) + token * 128;
          const uint4 c = kr[e];
          *reinterpret_cast<uint4*>(dst + (((2 * q) ^ (token & 7)) << 4)) =
              make_uint4(two_codes<false>(c.x), two_codes<true>(c.x), two_codes<false>(c.y), two_codes<true>(c.y));
          *reinterpret_cast<uint4*>(dst + (((2 * q + 1) ^ (token & 7)) << 4)) =
              make_uint4(two_codes<false>(c.z), two_codes<true>(c.z), two_codes<false>(c.w), two_codes<true>(c.w));
        }
        if (w == 0 && lane < BLOCKS) scales[it % SCALE_SLOTS][lane] = scale;
        fence_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(k_full + 8 * s);
          if (w == 0) mbar_arrive(sc_full + 8 * (it % SCALE_SLOTS));
        }
        fetch_k(place);
        if (!wait.all(v_empty + 8 * s, ph ^ 1u)) break;
        uint8_t* vt = tiles_at + TRACKS * C::Q_BYTES + (STAGES + s) * C::T_BYTES;
#pragma unroll
        for (int e = 0; e < V_EACH; ++e) {
          const int i = e * CODE_WARPS + w, blk = 2 * (i % (BLOCKS / 2)) + vb, c = i / (BLOCKS / 2);
          const uint4 lo = vr[2 * e], hi = vr[2 * e + 1];
          const uint32_t l4[4] = {lo.x, lo.y, lo.z, lo.w}, h4[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int row = 32 * c + 4 * vg + k;
            *reinterpret_cast<uint4*>(vt + blk / 4 * (P * 128) + row * 128 + (((2 * (blk & 3) + vu) ^ (row & 7)) << 4)) =
                make_uint4(two_codes<false>(l4[k]), two_codes<true>(l4[k]), two_codes<false>(h4[k]), two_codes<true>(h4[k]));
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_full + 8 * s);
        fetch_v(place);
        scale = next_scale;
      }
    }
  } else {
    fewer_registers<MMA_REGS>();
    if (warp == MMA_WARP) {
      uint32_t it = 0, n_piece = 0;
      bool ok = true;
      // scores of step i (of the line) of track x
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
      for (long long u = line_begin; ok && u < line_end; ++n_piece) {
        const Piece pc = piece(u);
        const long long stop = min(line_end, pc.end);
        u = max(u, pc.begin);
        if (u >= stop) break;
        const int steps = (int)(stop - u);
        u = stop;
        ok = wait.all(k_full + 8 * (it % STAGES), it / STAGES & 1u);
        for (int x = 0; x < TRACKS && ok; ++x) {
          ok = wait.all(q_full + 8 * x, n_piece & 1u);
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
            ok = wait.all(w_full + 8 * sb, TRACKS == 2 ? it & 1u : it >> 1 & 1u) && wait.all(v_full + 8 * s, it / STAGES & 1u);
            if (!ok) break;
            tc_fence_after();
            const uint64_t vd = make_kmajor_sw128_desc(v_at + s * C::T_BYTES);
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < TN / 16; ++k)
                tc_mma_f16_ts(tmem + C::O_COL + x * P, tmem + C::S_COL + sb * TN + 8 * k, desc_of(vd, k / 4 * (P * 128) + k % 4 * 32),
                              idesc_f16(P), j > 0 || k > 0);
              tc_commit(o_full + 8 * x);
              if (x == TRACKS - 1) tc_commit(v_empty + 8 * s);
            }
            __syncwarp();
            if (TRACKS == 2 && j + 1 < steps) {
              if (x == 0) ok = wait.all(k_full + 8 * ((it + 1) % STAGES), (it + 1) / STAGES & 1u);
              if (!ok) break;
              tc_fence_after();
              scores(it + 1, x);
            }
          }
        }
      }
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

template <int P>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t stream) {
  using C = Cfg<P>;
  const cudaError_t e = ensure_dynamic_smem((const void*)attend_many_kernel<P>, C::SMEM);
  if (e != cudaSuccess) return e;
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
