// Shared declarations of the kernels that keep keys and values in 8 bits and attend over them (admmq_cache.h).
#pragma once
#include <cuda_fp16.h>

#include "../../include/admmq_cache.h"
#include "adapt.h"

namespace admmq {

// Layout.  A block is 16 tokens of one page and head.  With P = head_dim rounded up to 64 (values past head_dim are never
// read), its 32 P bytes are the keys' codes, then the values', one byte code + 128 each:
//   keys    [P / 64][token 16][64]: value 64 h + e of a token at h * 1024 + token * 64 + e
//   values  [P / 32][g 8][t 4][i 4][4 tokens]: value 32 c + 4 g + i at c * 512 + g * 64 + t * 16 + i * 4 + {0, 1, 2, 3} for
//           tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
// so that lane 4 g + t of a warp finds in consecutive 16 bytes, and the warp in 512, what it feeds to m16n8k16 products as
// their second operand: of the keys 16 values of token g (or g + 8), of the values the four tokens of its rows of the
// product for four columns.  Blocks: [page][head][block of the page]; scales likewise, (key scale, value scale) each.
constexpr int CBLOCK = ADMMQ_CACHE_BLOCK;

struct CacheView {
  uint8_t* codes;
  float2* scale;
  int n_pages, heads, d, p;          // p = d rounded up to 64
  int bpp, bpp_shift;                // blocks of a page, log2 of that
  int block_bytes;                   // 32 p
};
// The rows of a call, as the device sees them.
struct PlanView {
  const int* tables;
  const int* held;
  const int4* blocks;                // (request, i, first row, rows): the i-th block that its rows touch, if they touch so many
  const int4* small;                 // tiles of packed rows: (request, first packed row, first row, rows of the request)
  const int4* big;
  int max_pages, group, n_blocks, n_small, n_big;
  int small_rows;                    // most packed rows that a small tile holds
  long long capacity;                // positions of a table
};
constexpr int FEW_ROWS = 16, MANY_ROWS = 256;   // packed rows (token, query head) of a tile

// Position of a request's first row; -1 where it takes no part.
__device__ __forceinline__ long long first_position(const PlanView& pl, int request, int rows, int* status) {
  const int at = pl.held[request];
  if (at < 0) return -1;
  if ((long long)at + rows > pl.capacity) {
    raise_status(status, ADMMQ_ERR_SHAPE);
    return -1;
  }
  return at;
}
// Index of block `b` (16 b = its first position) of a request and head 0; -1 for a page that does not exist.
__device__ __forceinline__ long long block_index(const CacheView& c, const PlanView& pl, int request, int b, int* status) {
  const int page = pl.tables[(long long)request * pl.max_pages + (b >> c.bpp_shift)];
  if ((unsigned)page >= (unsigned)c.n_pages) {
    raise_status(status, ADMMQ_ERR_SHAPE);
    return -1;
  }
  return (long long)page * c.heads * c.bpp + (b & c.bpp - 1);
}

// Codes of bytes 0, 1 (HIGH: 2, 3) of a word as two fp16 numbers.
template <bool HIGH>
__device__ __forceinline__ uint32_t two_codes(uint32_t w) {
  const uint32_t x = __byte_perm(w, 0x64646464u, HIGH ? 0x4342 : 0x4140);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Exponents of weights take log2 of the block's value scale, the sum of weights its reciprocal.  A block whose values are all zero
// (scale 0) adds nothing to the result, so it counts with a scale below any that a block can have (2^-40 / 127): its weights
// are in the sum as they should be, and never set a reference at which those of other blocks would have no bits left.
constexpr float LOG2_SCALE_OF_ZEROS = -47.0f, INV_SCALE_OF_ZEROS = 140737488355328.0f;   // 2^47
struct ValueScale {
  float log2, inv;
};
__device__ __forceinline__ ValueScale value_scale(float s) {
  if (s == 0.0f) return {LOG2_SCALE_OF_ZEROS, INV_SCALE_OF_ZEROS};
  // (no NaN for the sum of weights: a weight of NaN brings it by itself, and one that is not seen does not)
  return {__log2f(s), s == s ? __fdividef(1.0f, s) : 1.0f};
}

struct StoreArgs {
  CacheView c;
  PlanView pl;
  const void *k, *v;                 // write: rows;  read: outputs
  long long k_row, k_head, v_row, v_head;
  int* status;
};
cudaError_t launch_cache_write(const StoreArgs& a, bool is_bf16, cudaStream_t stream);
cudaError_t launch_cache_read(const StoreArgs& a, bool is_bf16, cudaStream_t stream);

// What is to be joined of a (tile, head): the CTAs first .. last have its parts; the same CTA twice: nothing.
struct __align__(16) Join {
  int first, last, head, row0;         // row0: packed row of the tile's first
  int first_row, rows, pad[2];         // first row of the request; packed rows of the tile
};
struct AttendArgs {
  CacheView c;
  PlanView pl;
  const bf16* q;
  bf16* out;
  float* lse;
  long long q_row, q_head, out_row, out_head;
  float scale_log2;                  // scale * log2(e)
  int window;
  int* status;
  // workspace of one kind of tiles: for every CTA two partial results, and what is to be joined
  float* part;                       // [ctas][2][rows][p]
  float2* part_ml;                   // [ctas][2][rows]: maximum (base 2) and sum
  Join* joins;
  int by_piece;                      // joins go by (tile, head), which are no more than CTAs; or by the first CTA
};
// CTAs of an SM that run attention of a few rows
__host__ __device__ constexpr int few_ctas(int p) { return p <= 64 ? 4 : p <= 128 ? 3 : 2; }
__host__ __device__ constexpr int many_rows(int p) { return p <= 128 ? MANY_ROWS : MANY_ROWS / 2; }
// CTAs of either kernel, and (tile, head)s.
inline int attend_ctas(int p, bool many, int sms) { return sms * (many ? 1 : few_ctas(p)); }
inline long long pieces_of(const AttendArgs& a, bool many) {
  return (long long)(many ? a.pl.n_big * (MANY_ROWS / many_rows(a.c.p)) : a.pl.n_small) * a.c.heads;
}
cudaError_t launch_cache_attend_few(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_cache_attend_many(const AttendArgs& a, cudaStream_t stream);
cudaError_t launch_cache_join(const AttendArgs& a, bool many, int sms, cudaStream_t stream);

}  // namespace admmq
