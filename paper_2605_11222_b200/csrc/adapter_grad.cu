// Gradients of the adapters:  G_a[r][c] = sum over the rows t of adapter a of f[t][r] v[t][c],
// once with (f, v) = (u, x) for down and once with (h, dy) for up, both in one launch.
//
// Bound: memory, the one pass over x (8 bits a value when it comes from a checkpoint) and dy; the factors f are rank
// values a row.  A CTA owns 128 columns (one checkpoint block) of one adapter and a share of its rows.  Rows arrive 64 at
// a time in registers, the next 64 on their way while these are multiplied (row numbers four tiles further), and become
// bf16 tiles [row][column] in one of two buffers, so that a tile costs one barrier; ldmatrix.trans turns those into
// operands of mma.sync: the contraction runs over the rows, so both operands are read across their storage order.
// Four CTAs a multiprocessor (rank 16) hide a tile's chain of arrival, conversion, barrier and products better than
// more tiles in flight in fewer CTAs: 8192 rows of 12288 (8 bits) + 4096 columns take 66 us, with four tiles ahead in two
// CTAs 84, with asynchronous copies to shared memory 129 (x in bf16 65 us); what is left is the way of every value through
// shared memory, which is 74 % busy, and the issue of some 200 instructions a warp and tile, 80 of them the conversion of
// codes.  (The tensor work, 2 rank flop a value read, is far below what mma.sync
// delivers: tcgen05 would wait for the same loads.)
// The shares of one (adapter, columns) tile form a cluster; their fp32 sums meet over distributed shared memory and
// are added in rank order, so nothing goes through global memory and the result does not depend on timing.
//
// Rounding.  x^ = scale code: the code (at most 127) is exact in bf16 and the scale is multiplied into f in fp32, so
// f scale is rounded once, as f is on the bf16 path: at most 2^-8 relative a term, the size of the output's own rounding.
#include <cooperative_groups.h>

#include "adapt.h"

namespace cg = cooperative_groups;

namespace admmq {
namespace {

constexpr int THREADS = 256;
constexpr int COLS = 128, ROWS = 64;
constexpr int IDS = 8;                               // tiles whose row numbers are kept, a power of two
constexpr int V_STRIDE = COLS + 8;                 // bf16; 272 bytes: eight rows of 16 bytes fall in eight bank groups

struct Side {
  const float* f;            // [T][rank]
  const bf16* v;             // [T][ldv] or NULL: codes
  long long ldv;
  const int8_t* codes;       // [T][width]
  const float* scale;        // [T][nb]
  bf16* grad;                // [n][rank][width]
  int width, nb;
};
struct GradParams {
  Side side[2];              // down, up
  int tiles0;                // column tiles of side 0
  const int* order;
  const int* offsets;
  long long T;
  int rank;
};

__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], const void* p) {
  const uint32_t a = (uint32_t)__cvta_generic_to_shared(p);
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}

// Two codes (bytes k and k + 1 of `c`, already offset by 128) as bf16: 2^23 + u minus 2^23 + 128 is exact.
template <int K>
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t c) {
  const float2 u = make_float2(__uint_as_float(__byte_perm(c, 0x4B000000u, 0x7540 + K)),
                               __uint_as_float(__byte_perm(c, 0x4B000000u, 0x7540 + K + 1)));
  const float2 v = __fadd2_rn(u, make_float2(-8388736.0f, -8388736.0f));
  return float2_to_bf16x2(v.x, v.y);
}

template <int MT>
struct Cfg {                                          // MT tiles of 16 ranks
  static constexpr int RP = 16 * MT, F_STRIDE = RP + 8;
  static constexpr int RESIDENT = MT == 1 ? 4 : MT == 2 ? 3 : MT == 4 ? 2 : 1;    // CTAs a multiprocessor holds
  static constexpr int BUF_BYTES = ROWS * (V_STRIDE + F_STRIDE) * 2, SUM_BYTES = RP * COLS * 4;
  static constexpr int IDS_AT = 2 * BUF_BYTES > SUM_BYTES ? 2 * BUF_BYTES : SUM_BYTES;
  static constexpr int BYTES = IDS_AT + IDS * ROWS * 4;
};

// One CTA's rows [lo + tile0 * ROWS, hi) of one adapter, EIGHT: v comes as codes and scales.
template <int MT, bool EIGHT>
__device__ __forceinline__ void accumulate(const GradParams& P, const Side& S, uint8_t* smem, int blk, long long lo,
                                           long long hi, long long tile0, long long tile1, float (&acc)[MT][2][4]) {
  using C = Cfg<MT>;
  constexpr int RP = C::RP, F_STRIDE = C::F_STRIDE;
  constexpr int FQ = ROWS * RP / 4 / THREADS;                     // pieces of 4 factors a thread: MT
  int* ids = reinterpret_cast<int*>(smem + C::IDS_AT);            // [IDS][ROWS] row numbers, -1: none
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int c0 = blk * COLS;
  // 16 threads a row of 8 columns each, 16 rows a pass
  const int vc = (tid & 15) * 8, vr = tid >> 4;
  const bool vin = c0 + vc < S.width;

  struct Tile {
    uint4 v[EIGHT ? ROWS / 32 : ROWS / 16];                       // (two rows of codes to a register quad)
    float4 f[FQ];
    float s[EIGHT ? FQ : 1];                                      // (multiplied when the tile is put down, not on arrival)
  };
  Tile reg;

  auto row_id = [&](long long tile, int row) -> int {
    const long long k = lo + tile * ROWS + row;
    if (tile >= tile1 || k >= hi) return -1;
    const int t = P.order[k];
    return (long long)t < P.T && t >= 0 ? t : -1;
  };
  auto load = [&](Tile& r, const int* id) {
#pragma unroll
    for (int q = 0; q < ROWS / 16; ++q) {
      const int t = id[vr + 16 * q];
      const bool in = t >= 0 && vin;
      if (EIGHT) {
        const uint2 c = in ? __ldg(reinterpret_cast<const uint2*>(S.codes + (long long)t * S.width + c0 + vc)) : make_uint2(0, 0);
        uint4& w = r.v[q >> 1];
        if (q & 1) {
          w.z = c.x;
          w.w = c.y;
        } else {
          w.x = c.x;
          w.y = c.y;
        }
      } else {
        r.v[EIGHT ? 0 : q] = in ? ldg_stream(S.v + (long long)t * S.ldv + c0 + vc) : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      const int i = tid + THREADS * q, row = i / (RP / 4), r4 = (i % (RP / 4)) * 4, t = id[row];
      const bool in = t >= 0 && r4 < P.rank;                      // rank is a multiple of 8
      r.f[q] = in ? __ldg(reinterpret_cast<const float4*>(S.f + (long long)t * P.rank + r4)) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (EIGHT) r.s[EIGHT ? q : 0] = in ? __ldg(S.scale + (long long)t * S.nb + blk) : 0.0f;
    }
  };
  auto put = [&](const Tile& r, bf16* vt, bf16* ft) {
#pragma unroll
    for (int q = 0; q < ROWS / 16; ++q) {
      uint4 o;
      if (EIGHT) {
        const uint4& w = r.v[q >> 1];
        const uint32_t a = ((q & 1) ? w.z : w.x) ^ 0x80808080u, b = ((q & 1) ? w.w : w.y) ^ 0x80808080u;   // + 128
        o = make_uint4(codes_to_bf16x2<0>(a), codes_to_bf16x2<2>(a), codes_to_bf16x2<0>(b), codes_to_bf16x2<2>(b));
      } else {
        o = r.v[EIGHT ? 0 : q];
      }
      *reinterpret_cast<uint4*>(vt + (vr + 16 * q) * V_STRIDE + vc) = o;
    }
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
      const int i = tid + THREADS * q, row = i / (RP / 4), r4 = (i % (RP / 4)) * 4;
      const float s = EIGHT ? r.s[EIGHT ? q : 0] : 1.0f;
      *reinterpret_cast<uint2*>(ft + row * F_STRIDE + r4) =
          make_uint2(float2_to_bf16x2(r.f[q].x * s, r.f[q].y * s), float2_to_bf16x2(r.f[q].z * s, r.f[q].w * s));
    }
  };

  // A row number is a load that the tile's loads wait for, so those of the next four tiles are in shared memory and the
  // ones after them on their way in a register of the first 64 threads.
  constexpr int KNOWN = THREADS / ROWS;
  static_assert(2 * KNOWN <= IDS, "row numbers put down meet no reader before a barrier");
  ids[tid] = row_id(tile0 + tid / ROWS, tid % ROWS);
  int next = 0;                                                   // tile to load next, from tile0
  int coming = tid < ROWS ? row_id(tile0 + KNOWN, tid) : -1;
  __syncthreads();
  auto advance = [&](Tile& r) {
    load(r, ids + (next & (IDS - 1)) * ROWS);                     // (past the last tile every row number is -1)
    if (tid < ROWS) {
      ids[((next + KNOWN) & (IDS - 1)) * ROWS + tid] = coming;
      coming = row_id(tile0 + next + KNOWN + 1, tid);
    }
    ++next;
  };
  advance(reg);
  int buf = 0;
  for (long long tile = tile0; tile < tile1; ++tile) {
    bf16* vt = reinterpret_cast<bf16*>(smem + buf * C::BUF_BYTES);          // [ROWS][V_STRIDE]
    bf16* ft = vt + ROWS * V_STRIDE;                                        // [ROWS][F_STRIDE]
    put(reg, vt, ft);
    __syncthreads();                                              // (and the buffer of two tiles ago is free)
    advance(reg);
#pragma unroll
    for (int r = 0; r < ROWS; r += 16) {
      uint32_t b[4];                                              // two tiles of 8 columns
      ldmatrix_x4_trans(b, vt + (r + (lane & 15)) * V_STRIDE + warp * 16 + (lane >> 4) * 8);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint32_t f[4];
        ldmatrix_x4_trans(f, ft + (r + (lane & 7) + (lane >> 4) * 8) * F_STRIDE + m * 16 + ((lane >> 3) & 1) * 8);
        mma_bf16(acc[m][0], f, b[0], b[1]);
        mma_bf16(acc[m][1], f, b[2], b[3]);
      }
    }
    buf ^= 1;
  }
  __syncthreads();
}

template <int MT>
__global__ void __launch_bounds__(THREADS, Cfg<MT>::RESIDENT) adapter_grad_kernel(const __grid_constant__ GradParams P) {
  extern __shared__ __align__(16) uint8_t smem[];
  float* sums = reinterpret_cast<float*>(smem);                   // [16 MT][COLS], after the last tile
  cg::cluster_group cluster = cg::this_cluster();
  const int share = blockIdx.x, shares = gridDim.x;
  const bool up = (int)blockIdx.y >= P.tiles0;
  const Side& S = P.side[up ? 1 : 0];
  const int blk = (int)blockIdx.y - (up ? P.tiles0 : 0);
  const int c0 = blk * COLS;
  const int a = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int vc = (tid & 15) * 8, vr = tid >> 4;
  const bool vin = c0 + vc < S.width;

  // this share's part of the adapter's rows, in whole tiles
  long long lo = min((long long)max(P.offsets[a], 0), P.T), hi = min((long long)max(P.offsets[a + 1], 0), P.T);
  if (hi < lo) hi = lo;
  const long long tiles = (hi - lo + ROWS - 1) / ROWS;
  const long long tile0 = tiles * share / shares, tile1 = tiles * (share + 1) / shares;

  float acc[MT][2][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[m][n][e] = 0.0f;
  if (tile0 < tile1) {
    if (S.v == nullptr)
      accumulate<MT, true>(P, S, smem, blk, lo, hi, tile0, tile1, acc);
    else
      accumulate<MT, false>(P, S, smem, blk, lo, hi, tile0, tile1, acc);
  }

  const int g = lane >> 2, q2 = (lane & 3) * 2;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int col = warp * 16 + n * 8 + q2;
      *reinterpret_cast<float2*>(sums + (m * 16 + g) * COLS + col) = make_float2(acc[m][n][0], acc[m][n][1]);
      *reinterpret_cast<float2*>(sums + (m * 16 + g + 8) * COLS + col) = make_float2(acc[m][n][2], acc[m][n][3]);
    }
  cluster.sync();
  // rank `share` of the cluster adds up every shares-th pair of ranks: 16 threads a row of 8 columns each
  for (int r = share * 16 + vr; r < P.rank; r += shares * 16) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.0f;
    for (int k = 0; k < shares; ++k) {
      const float* o = cluster.map_shared_rank(sums, k) + r * COLS + vc;
      const float4 x = *reinterpret_cast<const float4*>(o), y = *reinterpret_cast<const float4*>(o + 4);
      s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
      s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
    }
    if (vin) {
      uint4 o;
      o.x = float2_to_bf16x2(s[0], s[1]);
      o.y = float2_to_bf16x2(s[2], s[3]);
      o.z = float2_to_bf16x2(s[4], s[5]);
      o.w = float2_to_bf16x2(s[6], s[7]);
      *reinterpret_cast<uint4*>(S.grad + ((long long)a * P.rank + r) * S.width + c0 + vc) = o;
    }
  }
  cluster.sync();                                                 // no CTA leaves while its sums are read
}

template <int MT>
cudaError_t launch_mt(const GradParams& P, int tiles, int n, cudaStream_t stream) {
  constexpr int BYTES = Cfg<MT>::BYTES;
  const cudaError_t e = ensure_dynamic_smem((const void*)adapter_grad_kernel<MT>, BYTES);
  if (e != cudaSuccess) return e;
  // Shares of an adapter's rows: as many as the multiprocessors hold at once (a share starts with a chain of three loads,
  // so that more and shorter ones lose), while each keeps four tiles if the rows are spread evenly over the adapters;
  // at most the portable cluster.
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  int shares = 1;
  while (shares < 8 && (long long)tiles * n * 2 * shares <= (long long)Cfg<MT>::RESIDENT * sms &&
         P.T / n >= 4LL * ROWS * 2 * shares)
    shares *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(shares, tiles, n);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = shares;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, adapter_grad_kernel<MT>, P);
}

}  // namespace

cudaError_t launch_adapter_grad(const admmq_adapter_grad_args& a, cudaStream_t stream) {
  GradParams P = {};
  P.side[0] = {a.d_u, (const bf16*)a.d_x, a.ldx, (const int8_t*)a.d_x_codes, a.d_x_scale, (bf16*)a.d_grad_down, a.d_in,
               (a.d_in + ADMMQ_CHECKPOINT_BLOCK - 1) / ADMMQ_CHECKPOINT_BLOCK};
  P.side[1] = {a.d_h, (const bf16*)a.d_dy, a.lddy, nullptr, nullptr, (bf16*)a.d_grad_up, a.d_out, 0};
  P.tiles0 = (a.d_in + COLS - 1) / COLS;
  const int tiles = P.tiles0 + (a.d_out + COLS - 1) / COLS;
  P.order = a.d_order;
  P.offsets = a.d_offsets;
  P.T = a.n_rows;
  P.rank = a.rank;
  if (a.rank <= 16) return launch_mt<1>(P, tiles, a.n_adapters, stream);
  if (a.rank <= 32) return launch_mt<2>(P, tiles, a.n_adapters, stream);
  if (a.rank <= 64) return launch_mt<4>(P, tiles, a.n_adapters, stream);
  return launch_mt<8>(P, tiles, a.n_adapters, stream);
}

}  // namespace admmq
