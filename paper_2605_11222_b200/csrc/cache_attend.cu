// Attention of a few rows over the 8-bit cache: one new token of a request, or a few drafted ones.
//   z_j = scale q . k_j,  out = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m)
//
// Bound: reading the cache, once (128 requests of 6000 tokens, 32 query and 8 key heads of 128: 250 us, 6.3 TB/s), and
// issue, 47 % of the slots; short calls the 6 us before the first codes are there and the 5 us of the join.  A warp takes
// 32 positions (two blocks; one of heads of more than 128) at a time.  Their codes come as a bulk copy a block into a ring
// of its own in shared memory, in the order of the second operand of m16n8k16 products (16 bytes a lane, 512 a warp and
// load), while those before are worked on: 192 KB an SM.  (Codes loaded into registers a step ahead instead left room for
// eight warps an SM, which ran at 4.2 TB/s.)  The 16 rows of the product are the query heads of one key head, of one token
// or of several; where fewer are in use the product's other rows cost nothing that memory would not.
// Codes become fp16 by placing them in the mantissa of 1024 + (code + 128) and subtracting 1152: exact, two instructions
// for two.  Scales stay out of the products: the key scale multiplies the finished score, and the value scale s_b of a block
// enters the exponent, w_j = s_b exp(z_j - m') = 2^(z_j log2 e + log2 s_b - m'), with m' 10 to 15 below the running maximum of that
// exponent, so that fp16 holds w_j with 11 bits down to 2^-24 of the largest whatever the scales are, and the sum of weights takes
// w_j / s_b in fp32.
//
// Work is shared out in equal parts (cache_schedule.cuh); four warps of a CTA take turns through its units, each with a
// maximum, a sum and an accumulator of its own, joined in shared memory at the end of a piece.
#include "../../include/admmq_testing.h"
#include "cache_schedule.cuh"
#include "linear_tc.cuh"

namespace admmq {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS, LEAST_UNITS = WARPS, EXTRA = 12;
constexpr int MOST_RANKS = 16;                       // CTAs of a cluster
// Positions of a table for each of them, at most: a cluster is as slow as its longest request.  Heads of 128, 8 heads of keys,
// clusters / shared out: 27 requests of 2000 27 / 37 us, 50 of 1000 25 / 39, 6 of 8000 27 / 30, one of 16000 22 / 20; one of 2000
// among 26 of 60 tokens 19 / 15.
constexpr long long RANK_POSITIONS = 1024;
// Weights are fp16: the first largest of a row is 2^TOP, later ones stay below 2^LIMIT, so that weights down to 2^-24 of the largest
// have 11 bits, and those down to 2^-35 some.  (Behind a token with 99 % of the weight, a million positions of one size: the
// result is off by 23 % with TOP 0, 0.6 % with 6, by its own rounding with 10.  The time is the same: memory pays.)
constexpr float TOP = 10.0f, LIMIT = 15.0f;
constexpr float LN2 = 0.693147180559945309f;

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}

template <int P>
struct Few {
  static constexpr int NB = P <= 128 ? 2 : 1;                  // blocks of a step
  static constexpr int UNIT = NB * CBLOCK;
  static constexpr int BLOCK_BYTES = 2 * CBLOCK * P, UNIT_BYTES = NB * BLOCK_BYTES;   // codes of a block, of a step
  static constexpr int STAGES = P == 192 ? 4 : P == 256 || P == 64 ? 3 : 2;
  static constexpr int RING_BYTES = WARPS * STAGES * UNIT_BYTES;
  struct Shared {
    uint4 q[P / 16][32];                             // first operand: [64 h + 4 s .. of every 16][lane]
    Schedule<THREADS> schedule;
    long long total, line_end;                       // of the line, and where this CTA's part ends
    int ctas;                                        // that have a part
    float row_scale[FEW_ROWS];
    float m[WARPS][FEW_ROWS], l[WARPS][FEW_ROWS];
    int abort;
    Piece piece[2];                                  // the one at hand and the next, found once: all go by the same lengths
    uint64_t full[WARPS][STAGES];                    // a step's codes are there
  };
  static constexpr int O_ROW = P + 4;                // the warps' sums, [warp][row], over the rings once they are done
  static_assert(WARPS * FEW_ROWS * O_ROW * 4 + FEW_ROWS * (P * 4 + 8) <= RING_BYTES, "the sums lie over the rings");
  static constexpr int SMEM = RING_BYTES + (int)sizeof(Shared);
  static_assert((SMEM + 1024) * few_ctas(P) <= 228 * 1024, "shared memory");
};

struct FewArgs {
  AttendArgs a;
  long long wait_limit;
  int hold_loads;
};

// CLUSTER: the CTAs of a cluster share one (tile, head) and add up over distributed shared memory, so that there is nothing
// to find first and nothing to join after; for so few (tile, head)s that all their clusters run at once.
template <int P, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, few_ctas(P)) attend_few_kernel(const __grid_constant__ FewArgs A) {
  using F = Few<P>;
  constexpr int UNIT = F::UNIT, NB = F::NB;
  const AttendArgs& a = A.a;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  typename F::Shared& sh = *reinterpret_cast<typename F::Shared*>(smem_raw + F::RING_BYTES);
  float* const sums = reinterpret_cast<float*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int group = a.pl.group, heads = a.c.heads, d = a.c.d;
  uint8_t* const ring = smem_raw + warp * F::STAGES * F::UNIT_BYTES;
  const uint32_t ring_at = smem_u32(ring), full = smem_u32(&sh.full[warp][0]);
  if (lane == 0) {
    for (int i = 0; i < F::STAGES; ++i) mbar_init(full + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (tid == 0) sh.abort = 0;                        // (before the barriers of the schedule)
  const WarpWait wait = {&sh.abort, a.status, A.wait_limit};
  bool dead = false;                                 // a wait of this warp has run out: it does no more
  uint32_t issued = 0, taken = 0;                    // steps of this warp so far
  if (!CLUSTER) pdl_launch();                        // (the join; the next call, where there is none, gains nothing by being
  pdl_wait();                                        // there earlier: one token over 1000, calls in turn, 9.7 us, 9.2 so)
  if (CLUSTER) pdl_launch();

  const auto job = [&](int tile) { return __ldg(a.pl.small + tile); };
  const int cta = blockIdx.x;
  int rank = 0, ranks = 1;
  long long u = 0;
  if (CLUSTER) {
    rank = (int)cluster_ctarank();
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    if (tid == 0) {
      Piece& pc = sh.piece[0];
      sh.line_end = 1;
      pc.tile = cta / ranks / heads;
      pc.head = cta / ranks - pc.tile * heads;
      pc.job = job(pc.tile);
      pc.span = span_of(a, pc.job, FEW_ROWS);
      pc.begin = 0;
      pc.end = units_of<UNIT>(pc.span, pc.job, group);
    }
    __syncthreads();
  } else {
    const long long total = make_schedule<THREADS, UNIT, FEW_ROWS, EXTRA>(a, job, a.pl.n_small, sh.schedule) * heads;
    const int ctas = active_ctas(total, LEAST_UNITS);
    if (cta >= ctas) {
      if (tid == 0) tell_none(a, cta);
      return;
    }
    u = line_at(total, cta, ctas);
    const long long line_end = line_at(total, cta + 1, ctas);
    if (tid == 0) {
      sh.total = total;
      sh.ctas = ctas;
      sh.line_end = line_end;
    }
    // (a thread looks into its own segment: a search by one warp took 1.5 us)
    if (sh.schedule.sums[tid] * heads <= u && u < sh.schedule.sums[tid + 1] * heads)
      sh.piece[0] = piece_of<THREADS, UNIT, FEW_ROWS, EXTRA>(a, job, a.pl.n_small, sh.schedule, tid, u);
    __syncthreads();
  }
  int pieces = 0;                                    // of this CTA so far
  bool told = false;                                 // of a (tile, head) that others end

  while (u < sh.line_end) {
    const Piece& pc = sh.piece[pieces & 1];
    long long stop;
    if (CLUSTER) {
      u = pc.end * rank / ranks;
      stop = pc.end * (rank + 1) / ranks;            // (perhaps none)
    } else {
      stop = min(sh.line_end, pc.end);
      u = max(u, pc.begin);
      if (u >= stop) break;
      if (u == pc.begin) {
        told = stop < pc.end;
        if (tid == 0) tell_join(a, pc, FEW_ROWS, cta, told ? cta_of(pc.end - 1, sh.total, sh.ctas) : cta);
      }
    }
    const int request = pc.job.x, key_head = pc.head;

    // ---- queries: each row times a power of two that brings its largest value to [2^13, 2^14), as fp16
    {
      const int row0 = pc.job.y, nr = min(FEW_ROWS, pc.job.w * group - row0);
      const int r = tid >> 3, sub = tid & 7, pr = row0 + r, token = pr / group, head = pc.head * group + pr % group;
      const bf16* src = a.q + (long long)(pc.job.z + token) * a.q_row + head * a.q_head;
      uint2 raw[P / 32];
      uint32_t tops = 0;                             // magnitudes are in the order of their bits
#pragma unroll
      for (int j = 0; j < P / 32; ++j) {
        const int at = 4 * (sub + 8 * j);
        raw[j] = r < nr && at < d ? __ldg(reinterpret_cast<const uint2*>(src + at)) : make_uint2(0, 0);
        tops = __vmaxu2(tops, __vmaxu2(raw[j].x & 0x7fff7fffu, raw[j].y & 0x7fff7fffu));
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) tops = __vmaxu2(tops, __shfl_xor_sync(0xffffffffu, tops, o));
      const float top = __uint_as_float(min(max(tops << 16, tops & 0xffff0000u), 0x7f800000u));   // (infinity for NaN)
      float inv;
      const float up = pow2_scale_for(top, &inv);
#pragma unroll
      for (int j = 0; j < P / 32; ++j) {
        const int at = 4 * (sub + 8 * j);                // value 64 h + 16 t' + 4 s of the row
        const float2 x = bf16x2_to_float2(raw[j].x), y = bf16x2_to_float2(raw[j].y);
        uint32_t* dst = reinterpret_cast<uint32_t*>(&sh.q[(at >> 6) * 4 + ((at >> 2) & 3)][(r & 7) * 4 + ((at >> 4) & 3)]) + (r >> 3);
        dst[0] = pack_f16(x.x * up, x.y * up);
        dst[2] = pack_f16(y.x * up, y.y * up);
      }
      if (sub == 0) sh.row_scale[r] = top < INFINITY ? a.scale_log2 * inv : __int_as_float(0x7fc00000);
    }
    __syncthreads();
    const float f0 = sh.row_scale[g], f1 = sh.row_scale[g + 8];
    // the last position that rows g and g + 8 see
    const int here0 = pc.span.at + (pc.job.y + g) / group, here1 = pc.span.at + (pc.job.y + g + 8) / group;
    const int first_here = pc.span.at + pc.job.y / group, last_here = pc.span.hi - 1;

    float o[P / 8][4];
#pragma unroll
    for (int i = 0; i < P / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float m0 = 0.0f, m1 = 0.0f, l0 = 0.0f, l1 = 0.0f;
    int empty = 3;                                   // bits: rows g, g + 8 have seen nothing so far

    const int unit0 = (int)(u - pc.begin) + pc.span.lo / UNIT, unit1 = (int)(stop - pc.begin) + pc.span.lo / UNIT;
    const int n_blocks = (pc.span.hi + CBLOCK - 1) / CBLOCK;
    // pages of a step's blocks; -1: none there
    struct Pages {
      int p[NB];
    };
    auto look = [&](int unit) {
      Pages n;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int blk = NB * unit + b;
        n.p[b] = -1;
        if (unit < unit1 && blk < n_blocks) {
          n.p[b] = a.pl.tables[(long long)request * a.pl.max_pages + (blk >> a.c.bpp_shift)];
          if (n.p[b] < 0) n.p[b] = 0x7fffffff;       // (-1 is "none", not a page that does not exist)
        }
      }
      return n;
    };
    // A step under way: its blocks' scales, and whether they exist.
    struct Step {
      float2 s[NB];
      bool exists[NB];
    };
    auto fetch = [&](int unit, const Pages& n) {
      Step f;
      int at[NB], bytes = 0;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int blk = NB * unit + b;
        f.exists[b] = (unsigned)n.p[b] < (unsigned)a.c.n_pages;
        if (n.p[b] >= a.c.n_pages) raise_status(a.status, ADMMQ_ERR_SHAPE);
        at[b] = f.exists[b] ? (n.p[b] * heads + key_head) * a.c.bpp + (blk & a.c.bpp - 1) : 0;
        bytes += f.exists[b] ? F::BLOCK_BYTES : 0;
        f.s[b] = f.exists[b] ? __ldg(a.c.scale + at[b]) : make_float2(0.f, 0.f);
      }
      if (unit < unit1) {
        if (lane == 0 && !A.hold_loads) {
          const uint32_t stage = issued % F::STAGES, bar = full + 8 * stage, dst = ring_at + stage * F::UNIT_BYTES;
          if (bytes) mbar_expect_tx(bar, bytes);
          else mbar_arrive(bar);
#pragma unroll
          for (int b = 0; b < NB; ++b)
            if (f.exists[b])
              bulk_load(dst + b * F::BLOCK_BYTES, a.c.codes + (size_t)(uint32_t)at[b] * (uint32_t)F::BLOCK_BYTES, F::BLOCK_BYTES, bar);
        }
        ++issued;
      }
      return f;
    };

    // the steps under way, in their order, and the pages of the one after
    Step ahead[F::STAGES];
    int unit = dead ? unit1 : unit0 + warp;
    {
      Pages n[F::STAGES];
#pragma unroll
      for (int i = 0; i < F::STAGES; ++i) n[i] = look(unit + i * WARPS);
      // (of the first step, blocks behind the window are not asked for: their pages may be gone)
#pragma unroll
      for (int b = 0; b + 1 < NB; ++b)
        if (NB * unit + b < pc.span.lo / CBLOCK) n[0].p[b] = -1;
#pragma unroll
      for (int i = 0; i < F::STAGES; ++i) ahead[i] = fetch(unit + i * WARPS, n[i]);
    }
    Pages next = look(unit + F::STAGES * WARPS);
    if (!CLUSTER && tid == THREADS - 1 && stop < sh.line_end)   // (while the copies are under way)
      sh.piece[~pieces & 1] = piece_after<UNIT, FEW_ROWS, EXTRA>(a, job, a.pl.n_small, sh.piece[pieces & 1]);
    for (; unit < unit1; unit += WARPS) {
      const uint32_t stage = taken % F::STAGES;
      dead = !wait.all(full + 8 * stage, taken / F::STAGES & 1u);
      if (dead) break;
      ++taken;
      const uint8_t* codes = ring + stage * F::UNIT_BYTES + lane * 16;
      // ---- scores of the step's positions
      float z[NB][2][4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j) z[b][j][0] = z[b][j][1] = z[b][j][2] = z[b][j][3] = 0.0f;
#pragma unroll
      for (int h = 0; h < P / 64; ++h) {
        uint4 k[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j) k[b][j] = *reinterpret_cast<const uint4*>(codes + b * F::BLOCK_BYTES + (2 * h + j) * 512);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const uint4 q = sh.q[h * 4 + s][lane];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint4& w = k[b][j];
              const uint32_t c = s == 0 ? w.x : s == 1 ? w.y : s == 2 ? w.z : w.w;
              mma_f16(z[b][j], q, two_codes<false>(c), two_codes<true>(c));
            }
        }
      }
      float2 sc[NB];
      bool exists[NB], all = true;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        sc[b] = ahead[0].s[b];
        exists[b] = ahead[0].exists[b];
        all &= exists[b];
      }
      // ---- exponents, base 2
      const int pos = unit * UNIT;
      const bool whole = pos + UNIT - 1 <= first_here && (a.window <= 0 || pos > last_here - a.window) && all;
      float most0 = -INFINITY, most1 = -INFINITY, inv_s[NB];   // of this lane's four positions of a block
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const ValueScale vs = value_scale(sc[b].y);
        const float lv = vs.log2, k0 = f0 * sc[b].x, k1 = f1 * sc[b].x;
        inv_s[b] = vs.inv;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            z[b][j][e] = fmaf(z[b][j][e], k0, lv - m0);
            z[b][j][2 + e] = fmaf(z[b][j][2 + e], k1, lv - m1);
            if (!whole) {
              const int p = pos + 16 * b + 8 * j + 2 * t + e;
              if (!exists[b] || p > here0 || (a.window > 0 && p <= here0 - a.window)) z[b][j][e] = -INFINITY;
              if (!exists[b] || p > here1 || (a.window > 0 && p <= here1 - a.window)) z[b][j][2 + e] = -INFINITY;
            }
            most0 = fmaxf(most0, z[b][j][e]);
            most1 = fmaxf(most1, z[b][j][2 + e]);
          }
        }
      }
      // The reference lies TOP below the row's maximum over the first positions seen; it is raised only where a weight would
      // pass 2^LIMIT, which is rare.
      if (__any_sync(0xffffffffu, empty || fmaxf(most0, most1) > LIMIT)) {
#pragma unroll
        for (int x = 1; x < 4; x <<= 1) {
          most0 = fmaxf(most0, __shfl_xor_sync(0xffffffffu, most0, x));
          most1 = fmaxf(most1, __shfl_xor_sync(0xffffffffu, most1, x));
        }
        const float by0 = (empty & 1 ? most0 > -INFINITY : most0 > LIMIT) ? most0 - TOP : 0.0f;
        const float by1 = (empty & 2 ? most1 > -INFINITY : most1 > LIMIT) ? most1 - TOP : 0.0f;
        // (where nothing was seen yet the sums are 0)
        const float a0 = empty & 1 ? 0.0f : exp2_fast(-by0), a1 = empty & 2 ? 0.0f : exp2_fast(-by1);
        if (most0 > -INFINITY) empty &= ~1;
        if (most1 > -INFINITY) empty &= ~2;
        m0 += by0;
        m1 += by1;
        l0 *= a0;
        l1 *= a1;
#pragma unroll
        for (int i = 0; i < P / 8; ++i) {
          o[i][0] *= a0;
          o[i][1] *= a0;
          o[i][2] *= a1;
          o[i][3] *= a1;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              z[b][j][e] -= by0;
              z[b][j][2 + e] -= by1;
            }
      }
      uint4 w[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            z[b][j][e] = exp2_fast(z[b][j][e]);
            z[b][j][2 + e] = exp2_fast(z[b][j][2 + e]);
            s0 += z[b][j][e];
            s1 += z[b][j][2 + e];
          }
        }
        l0 = fmaf(s0, inv_s[b], l0);
        l1 = fmaf(s1, inv_s[b], l1);
        w[b] = make_uint4(pack_f16(z[b][0][0], z[b][0][1]), pack_f16(z[b][0][2], z[b][0][3]), pack_f16(z[b][1][0], z[b][1][1]),
                          pack_f16(z[b][1][2], z[b][1][3]));
      }
      // ---- values
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < P / 32; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(codes + b * F::BLOCK_BYTES + 16 * P + c * 512);
          mma_f16(o[4 * c], w[b], two_codes<false>(x.x), two_codes<true>(x.x));
          mma_f16(o[4 * c + 1], w[b], two_codes<false>(x.y), two_codes<true>(x.y));
          mma_f16(o[4 * c + 2], w[b], two_codes<false>(x.z), two_codes<true>(x.z));
          mma_f16(o[4 * c + 3], w[b], two_codes<false>(x.w), two_codes<true>(x.w));
        }
      __syncwarp();                                  // (every lane has read the stage)
#pragma unroll
      for (int i = 0; i + 1 < F::STAGES; ++i) ahead[i] = ahead[i + 1];
      ahead[F::STAGES - 1] = fetch(unit + F::STAGES * WARPS, next);
      next = look(unit + (F::STAGES + 1) * WARPS);
    }
    if (dead && !A.hold_loads)                       // copies in flight land before the memory is used again
      for (; taken != issued; ++taken) mbar_wait_quiet(full + 8 * (taken % F::STAGES), taken / F::STAGES & 1u);
    __syncthreads();                                 // (the sums go over every warp's ring)

    // ---- the warps' sums into one
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, x);
      l1 += __shfl_xor_sync(0xffffffffu, l1, x);
    }
    if (t == 0) {
      sh.m[warp][g] = empty & 1 ? -INFINITY : m0;
      sh.m[warp][g + 8] = empty & 2 ? -INFINITY : m1;
      sh.l[warp][g] = l0;
      sh.l[warp][g + 8] = l1;
    }
#pragma unroll
    for (int c = 0; c < P / 32; ++c)
#pragma unroll
      for (int half = 0; half < 2; ++half)           // columns 32 c + 8 t + 4 half + i of rows g and g + 8
#pragma unroll
        for (int r = 0; r < 2; ++r)
          *reinterpret_cast<float4*>(sums + (warp * FEW_ROWS + g + 8 * r) * F::O_ROW + 32 * c + 8 * t + 4 * half) =
              make_float4(o[4 * c][2 * r + half], o[4 * c + 1][2 * r + half], o[4 * c + 2][2 * r + half], o[4 * c + 3][2 * r + half]);
    __syncthreads();
    const int row0 = pc.job.y, nr = min(FEW_ROWS, pc.job.w * group - row0);
    const bool complete = !CLUSTER && u == pc.begin && stop == pc.end;
    float* const shared_o = sums + WARPS * FEW_ROWS * F::O_ROW;              // of a cluster's CTA: its sums, then its maxima
    float2* const shared_ml = reinterpret_cast<float2*>(shared_o + FEW_ROWS * P);
    const int slot = 2 * cta + (u == pc.begin ? 1 : 0);
    auto put = [&](int r, int at4, const float4& acc, float m, float l) {    // four values of a finished row
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const int pr = row0 + r, head = pc.head * group + pr % group;
      const long long row = pc.job.z + pr / group;
      *reinterpret_cast<uint2*>(a.out + row * a.out_row + head * a.out_head + at4) =
          make_uint2(float2_to_bf16x2(acc.x * inv, acc.y * inv), float2_to_bf16x2(acc.z * inv, acc.w * inv));
      if (at4 == 0 && a.lse) a.lse[row * (heads * group) + head] = l == 0.0f ? -INFINITY : m * LN2 + logf(l);
    };
    for (int i = tid; i < FEW_ROWS * P / 4; i += THREADS) {
      const int r = i / (P / 4), at4 = 4 * (i % (P / 4));
      if (r >= nr || at4 >= d) continue;
      float m = sh.m[0][r];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) m = fmaxf(m, sh.m[w][r]);
      const float ref = m == -INFINITY ? 0.0f : m;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.0f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float k = exp2_fast(sh.m[w][r] - ref);
        const float4 x = *reinterpret_cast<const float4*>(sums + (w * FEW_ROWS + r) * F::O_ROW + at4);
        acc.x = fmaf(x.x, k, acc.x);
        acc.y = fmaf(x.y, k, acc.y);
        acc.z = fmaf(x.z, k, acc.z);
        acc.w = fmaf(x.w, k, acc.w);
        l = fmaf(sh.l[w][r], k, l);
      }
      if (CLUSTER) {
        *reinterpret_cast<float4*>(shared_o + r * P + at4) = acc;
        if (at4 == 0) shared_ml[r] = make_float2(m, l);
      } else if (complete) {
        put(r, at4, acc, m, l);
      } else {
        *reinterpret_cast<float4*>(a.part + ((long long)slot * FEW_ROWS + r) * P + at4) = acc;
        if (at4 == 0) a.part_ml[slot * FEW_ROWS + r] = make_float2(m, l);
      }
    }
    if (CLUSTER) {
      cluster_sync_all();
      const uint32_t o_at = smem_u32(shared_o), ml_at = smem_u32(shared_ml);
      for (int i = rank * THREADS + tid; i < nr * (P / 4); i += ranks * THREADS) {
        const int r = i / (P / 4), at4 = 4 * (i % (P / 4));
        if (at4 >= d) continue;
        float m = -INFINITY, l = 0.0f;
        for (int k = 0; k < ranks; ++k) m = fmaxf(m, ld_cluster_f2(map_to_cta(ml_at + 8 * r, k)).x);
        const float ref = m == -INFINITY ? 0.0f : m;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < ranks; ++k) {
          const float2 ml = ld_cluster_f2(map_to_cta(ml_at + 8 * r, k));
          const float4 x = ld_cluster_f4(map_to_cta(o_at + (r * P + at4) * 4, k));
          const float f = exp2_fast(ml.x - ref);
          acc.x = fmaf(x.x, f, acc.x);
          acc.y = fmaf(x.y, f, acc.y);
          acc.z = fmaf(x.z, f, acc.z);
          acc.w = fmaf(x.w, f, acc.w);
          l = fmaf(ml.y, f, l);
        }
        put(r, at4, acc, m, l);
      }
      cluster_sync_all();                            // (a CTA's memory is read until here)
      return;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (copies go over the sums next)
    __syncthreads();
    u = stop;
    ++pieces;
  }
  if (tid == 0 && !told) tell_none(a, cta);
}

// Clusters of `ranks` CTAs (a power of two) that run at once on the current device; 0 on error.
template <int P>
int clusters_at_once(int ranks) {
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES][MOST_RANKS + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  std::atomic<int>& slot = known[dev][ranks];
  int n = slot.load(std::memory_order_relaxed);
  if (n == 0) {
    const void* kernel = (const void*)attend_few_kernel<P, true>;
    if (ensure_dynamic_smem(kernel, Few<P>::SMEM) != cudaSuccess) return 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ranks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Few<P>::SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, (const void*)attend_few_kernel<P, true>, &cfg) != cudaSuccess) return 0;
    if (n < 1) n = -1;
    slot.store(n, std::memory_order_relaxed);
  }
  return n;
}

template <int P>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t stream) {
  const long long pieces = pieces_of(a, false);
  int ranks = MOST_RANKS;                            // as many as leave every cluster running at once
  while (ranks > 0 && pieces > clusters_at_once<P>(ranks)) ranks /= 2;
  if (a.pl.capacity > ranks * RANK_POSITIONS) ranks = 0;
  const void* kernel = ranks > 0 ? (const void*)attend_few_kernel<P, true> : (const void*)attend_few_kernel<P, false>;
  const cudaError_t e = ensure_dynamic_smem(kernel, Few<P>::SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks > 0 ? (unsigned)(pieces * ranks) : attend_ctas(P, false, sms));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Few<P>::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ranks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ranks > 0 ? 2 : 1;
  const FewArgs args = {a, g_linear_wait_limit.load(std::memory_order_relaxed), g_linear_hold_loads.load(std::memory_order_relaxed)};
  if (ranks > 0) return cudaLaunchKernelEx(&cfg, attend_few_kernel<P, true>, args);
  const cudaError_t f = cudaLaunchKernelEx(&cfg, attend_few_kernel<P, false>, args);
  return f == cudaSuccess ? launch_cache_join(a, false, sms, stream) : f;
}

}  // namespace

cudaError_t launch_cache_attend_few(const AttendArgs& a, cudaStream_t stream) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  switch (a.c.p / 64) {
    case 1: return launch<64>(a, sms, stream);
    case 2: return launch<128>(a, sms, stream);
    case 3: return launch<192>(a, sms, stream);
    default: return launch<256>(a, sms, stream);
  }
}

}  // namespace admmq
