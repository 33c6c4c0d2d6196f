// Rows of keys and values into the 8-bit cache, and out of it.
//
// A warp holds one block (16 tokens of a head) of keys or of values: the rows that the call adds to it, read once, are in
// registers when their largest magnitude is known, and the codes leave in the order in which the cache keeps them, 16
// bytes a lane.  Where the block is held in part, the bytes of the earlier tokens are read, rounded to the new scale if it
// has grown, and written back.
// Bound: memory for many rows (a bf16 value is read as 2 bytes and written as 1; 65536 rows, 8 heads of 128: written in 76 us,
// 5.3 TB/s, read back in 73 us, 5.5 TB/s; in fp32 115 us, 5.8 TB/s, and 142, 4.7; 16384 rows, from and to cold memory, 29 and 25 us,
// where the ends count: a warp loads, works, then stores, with nothing under way meanwhile), a chain of latencies for
// one: position, page, row with held codes, maximum, store (a token of each of 77 requests, 4.4 us).
#include "cache.h"

namespace admmq {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS, ENOUGH_CTAS = 16;   // CTAs an SM that keep it busy
constexpr float LEAST = 9.094947017729282e-13f;     // 2^-40: magnitudes of a block that is held as zeros stay below
constexpr uint32_t MOST_BITS = 0x53800000u;         // 2^40

template <bool BF16, int N>
__device__ __forceinline__ void store_values(void* p, const float (&v)[N]) {
  if (BF16) {
    uint32_t r[N / 2];
#pragma unroll
    for (int e = 0; e < N / 2; ++e) r[e] = float2_to_bf16x2(v[2 * e], v[2 * e + 1]);
    if (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N / 8; ++i)
        *((uint4*)p + i) = make_uint4(r[(4 * i) % (N / 2)], r[(4 * i + 1) % (N / 2)], r[(4 * i + 2) % (N / 2)], r[(4 * i + 3) % (N / 2)]);
    } else {
      *(uint2*)p = make_uint2(r[0], r[1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) *((float4*)p + i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  }
}

// code + 128 in the low bytes, of two values.  The quotients as a division rounds them, from the reciprocal y of s: q0 =
// RN(x y), RN(q0 + (x - q0 s) y) (Markstein 1990); s is 0 (y is then 0 too, and the code 128) or at least 2^-47, and |x|
// below 2^40, so nothing overflows and no remainder underflows that could decide a rounding.  Adding 1.5 * 2^23 rounds to a
// whole number, ties to even, and leaves it in the low bits.  (Where the scale is NaN the code is any.)
struct Divisor {
  float2 y, minus_s;
};
__device__ __forceinline__ uint2 codes_of(float2 x, const Divisor& by) {
  const float2 q0 = __fmul2_rn(x, by.y), magic = make_float2(12583040.0f, 12583040.0f);
  const float2 t = __fadd2_rn(__ffma2_rn(__ffma2_rn(q0, by.minus_s, x), by.y, q0), magic);
  return make_uint2(__float_as_uint(t.x), __float_as_uint(t.y));
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ float value_of(uint32_t word, int byte) {   // code of a byte, exactly
  return __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7540u + byte)) - 8388736.0f;
}
// A byte's code at the new scale; r = old scale / new scale.
__device__ __forceinline__ uint32_t rounded_again(uint32_t word, int byte, float r) {
  return __float_as_uint(__fadd_rn(__fmul_rn(value_of(word, byte), r), 12583040.0f));
}

// What a CTA has to do: block b of a request, of which slots [first, first + n) are rows row .. of the call; its warps take
// keys and values of the heads in turns (a warp that looked the block up for one of them alone spent most of its time on
// that).
struct Unit {
  long long index;                   // of the block for head 0
  long long row;
  int first, n;
};
__device__ __forceinline__ bool find_unit(const StoreArgs& a, Unit& u) {
  const int4 job = __ldg(a.pl.blocks + blockIdx.x);
  const int row0 = job.z, rows = job.w;
  const long long at = first_position(a.pl, job.x, rows, a.status);
  if (at < 0) return false;
  const int b = (int)(at / CBLOCK) + job.y, begin = max((int)at, b * CBLOCK), end = min((int)at + rows, (b + 1) * CBLOCK);
  if (begin >= end) return false;
  u.index = block_index(a.c, a.pl, job.x, b, a.status);
  u.first = begin - b * CBLOCK;
  u.n = end - begin;
  u.row = row0 + (begin - at);
  return u.index >= 0;
}
// Keys (which even) or values (odd) of a head of the block.
struct Item {
  bool values;
  int head;
  uint8_t* block;
  float* scale;
  char* rows;                        // of the unit's first row
  long long row_bytes;
};
template <int E>
__device__ __forceinline__ Item item_of(const StoreArgs& a, const Unit& u, int which) {
  Item i;
  i.values = which & 1;
  i.head = which >> 1;
  const long long index = u.index + (long long)i.head * a.c.bpp;
  i.block = a.c.codes + index * a.c.block_bytes + (i.values ? 16 * a.c.p : 0);
  i.scale = &a.c.scale[index].x + (i.values ? 1 : 0);
  i.row_bytes = (i.values ? a.v_row : a.k_row) * E;
  i.rows = (char*)(i.values ? a.v : a.k) + u.row * i.row_bytes + i.head * (i.values ? a.v_head : a.k_head) * E;
  return i;
}

// CTAs of an SM that registers are limited for: more would spill, fewer leave the memory waiting (16384 rows, 8 heads of 128, bf16,
// again and again, in part from the L2 cache: 20.8 us with 6, 22.8 with 5 or 7, 24.5 without a limit; read back 18.6 with 8, 20.7
// without).
constexpr int write_ctas(bool bf16, int pc) { return bf16 ? (pc <= 2 ? 6 : 4) : pc == 1 ? 6 : pc == 2 ? 4 : 2; }
constexpr int read_ctas(int pc) { return pc <= 2 ? 8 : 5; }

// PC: the block's 64-value columns; the lane's share of them.
template <bool BF16, int PC>
__global__ void __launch_bounds__(THREADS, write_ctas(BF16, PC)) cache_write_kernel(const __grid_constant__ StoreArgs a) {
  Unit u;
  pdl_wait();
  if (!find_unit(a, u)) return;
  const int lane = threadIdx.x & 31, d = a.c.d;
  constexpr int E = BF16 ? 2 : 4;
  for (int which = blockIdx.y * WARPS + (threadIdx.x >> 5); which < 2 * a.c.heads; which += gridDim.y * WARPS) {
    const Item item = item_of<E>(a, u, which);
    const bool values = item.values;
    uint8_t* const block = item.block;
    const char* const x = item.rows;
    const long long row_bytes = item.row_bytes;
    const float held = u.first > 0 ? *item.scale : 0.0f;

    // The lane's rows as they are: of chunk o 16 values of one token (keys), or 4 of each of four tokens (values).
    constexpr int R = BF16 ? 8 : 16;
    uint32_t raw[2 * PC][R];
    uint32_t top = 0;
#pragma unroll
    for (int o = 0; o < 2 * PC; ++o) {
      if (!values) {
        const int slot = (lane >> 2) + 8 * (o & 1), at = (o >> 1) * 64 + (lane & 3) * 16;
        const bool on = slot >= u.first && slot < u.first + u.n && at < d;
        const uint4* src = reinterpret_cast<const uint4*>(x + (slot - u.first) * row_bytes + at * E);
#pragma unroll
        for (int i = 0; i < R / 4; ++i) {
          const uint4 w = on ? ldg_stream(src + i) : make_uint4(0, 0, 0, 0);
          raw[o][4 * i] = w.x;
          raw[o][4 * i + 1] = w.y;
          raw[o][4 * i + 2] = w.z;
          raw[o][4 * i + 3] = w.w;
        }
      } else {
        const int at = o * 32 + (lane >> 2) * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int slot = 2 * (lane & 3) + (k & 1) + 8 * (k >> 1);
          const bool on = slot >= u.first && slot < u.first + u.n && at < d;
          const char* src = x + (slot - u.first) * row_bytes + at * E;
          if (BF16) {
            const uint2 w = on ? __ldg(reinterpret_cast<const uint2*>(src)) : make_uint2(0, 0);
            raw[o][2 * k] = w.x;
            raw[o][2 * k + 1] = w.y;
          } else {
            const uint4 w = on ? __ldg(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
            raw[o][(4 * k) % R] = w.x;
            raw[o][(4 * k + 1) % R] = w.y;
            raw[o][(4 * k + 2) % R] = w.z;
            raw[o][(4 * k + 3) % R] = w.w;
          }
        }
      }
    }
    // codes of earlier tokens, if the block goes on
    uint4 old[2 * PC];
    if (u.first > 0) {
#pragma unroll
      for (int o = 0; o < 2 * PC; ++o)
        old[o] = *reinterpret_cast<const uint4*>(block + (values ? o * 512 + lane * 16 : (o >> 1) * 1024 + (o & 1) * 512 + lane * 16));
    }
    // (the order of the bit patterns is that of the magnitudes, with infinity and NaN on top)
#pragma unroll
    for (int o = 0; o < 2 * PC; ++o)
#pragma unroll
      for (int i = 0; i < R; ++i) top = BF16 ? __vmaxu2(top, raw[o][i] & 0x7fff7fffu) : max(top, raw[o][i] & 0x7fffffffu);
    if (BF16) top = max(top << 16, top & 0xffff0000u);
    top = __reduce_max_sync(0xffffffffu, top);
    const float most = __uint_as_float(top);
    const bool bad = top >= MOST_BITS || held != held;
    const float add = most < LEAST ? 0.0f : __fmul_rn(most, 1.0f / 127.0f);
    const float s = bad ? __int_as_float(0x7fc00000) : fmaxf(held, add);
    const bool zeros = bad || s == 0.0f;
    const float y = zeros ? 0.0f : __frcp_rn(s), r = zeros ? 0.0f : __fdiv_rn(held, s);
    const Divisor by = {make_float2(y, y), zeros ? make_float2(0.f, 0.f) : make_float2(-s, -s)};
    const bool again = u.first > 0 && !(s == held);  // earlier tokens are rounded again
    if (lane == 0) *item.scale = s;

    // values 2 i and 2 i + 1 of a chunk
    auto pair = [&](const uint32_t (&w)[R], int i) {
      return BF16 ? bf16x2_to_float2(w[i % R]) : make_float2(__uint_as_float(w[(2 * i) % R]), __uint_as_float(w[(2 * i + 1) % R]));
    };
#pragma unroll
    for (int o = 0; o < 2 * PC; ++o) {
      if (!values) {
        const int slot = (lane >> 2) + 8 * (o & 1), at = (o >> 1) * 64 + (lane & 3) * 16;
        uint4* dst = reinterpret_cast<uint4*>(block + (o >> 1) * 1024 + slot * 64 + (lane & 3) * 16);
        if (at >= d) continue;
        if (slot >= u.first && slot < u.first + u.n) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint2 k = codes_of(pair(raw[o], 2 * i), by), l = codes_of(pair(raw[o], 2 * i + 1), by);
            w[i] = pack4(k.x, k.y, l.x, l.y);
          }
          *dst = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (slot < u.first && again) {
          uint32_t w[4] = {old[o].x, old[o].y, old[o].z, old[o].w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = pack4(rounded_again(w[i], 0, r), rounded_again(w[i], 1, r), rounded_again(w[i], 2, r), rounded_again(w[i], 3, r));
          *dst = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
        const int at = o * 32 + (lane >> 2) * 4, low = 2 * (lane & 3);
        uint4* dst = reinterpret_cast<uint4*>(block + o * 512 + lane * 16);
        if (at >= d) continue;
        // codes of token k's four values, then the words of four tokens
        uint2 c[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          c[k][0] = codes_of(pair(raw[o], 2 * k), by);
          c[k][1] = codes_of(pair(raw[o], 2 * k + 1), by);
        }
        uint32_t w[4] = {pack4(c[0][0].x, c[1][0].x, c[2][0].x, c[3][0].x), pack4(c[0][0].y, c[1][0].y, c[2][0].y, c[3][0].y),
                         pack4(c[0][1].x, c[1][1].x, c[2][1].x, c[3][1].x), pack4(c[0][1].y, c[1][1].y, c[2][1].y, c[3][1].y)};
        if (u.first > 0) {                           // bytes of earlier tokens, rounded again or not, go in
          uint32_t mine = 0, before = 0;             // masks of the call's tokens, of the earlier ones
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int slot = low + (k & 1) + 8 * (k >> 1);
            if (slot < u.first) before |= 0xffu << (8 * k);
            else if (slot < u.first + u.n) mine |= 0xffu << (8 * k);
          }
          if (!mine && !(before && again)) continue;
          const uint32_t had[4] = {old[o].x, old[o].y, old[o].z, old[o].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t kept = again ? pack4(rounded_again(had[i], 0, r), rounded_again(had[i], 1, r), rounded_again(had[i], 2, r),
                                                rounded_again(had[i], 3, r))
                                        : had[i];
            w[i] = (w[i] & mine) | (kept & before) | (had[i] & ~(mine | before));
          }
        }
        *dst = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

template <bool BF16, int PC>
__global__ void __launch_bounds__(THREADS, read_ctas(PC)) cache_read_kernel(const __grid_constant__ StoreArgs a) {
  Unit u;
  pdl_wait();
  const int lane = threadIdx.x & 31, d = a.c.d;
  constexpr int E = BF16 ? 2 : 4;
  const bool found = find_unit(a, u);
  for (int which = blockIdx.y * WARPS + (threadIdx.x >> 5); which < 2 * a.c.heads; which += gridDim.y * WARPS) {
    if (!found) {
      // rows of a request that takes no part, or of a page that does not exist, read as zero
      const int4 job = __ldg(a.pl.blocks + blockIdx.x);
      const int row0 = job.z, rows = job.w;
      const int at = a.pl.held[job.x];
      int begin = 0, end = 0;
      if (at < 0 || (long long)at + rows > a.pl.capacity) {
        begin = CBLOCK * job.y;
        end = min(rows, begin + CBLOCK);
      } else {
        const int b = at / CBLOCK + job.y;
        begin = max(0, b * CBLOCK - at);
        end = min(rows, (b + 1) * CBLOCK - at);
      }
      u.index = 0;
      u.row = row0 + begin;
      const Item item = item_of<E>(a, u, which);
      for (int i = begin; i < end; ++i)
        for (int e = lane; e < d * E / 4; e += 32) reinterpret_cast<uint32_t*>(item.rows + (i - begin) * item.row_bytes)[e] = 0u;
      continue;
    }
    const Item item = item_of<E>(a, u, which);
    const bool values = item.values;
    const uint8_t* const block = item.block;
    const float s = *item.scale;
    char* const x = item.rows;
    const long long row_bytes = item.row_bytes;
    uint4 w[2 * PC];
#pragma unroll
    for (int o = 0; o < 2 * PC; ++o) {
      const int at = values ? o * 32 + (lane >> 2) * 4 : (o >> 1) * 64 + (lane & 3) * 16;
      const int off = values ? o * 512 + lane * 16 : (o >> 1) * 1024 + ((lane >> 2) + 8 * (o & 1)) * 64 + (lane & 3) * 16;
      if (at < d) w[o] = *reinterpret_cast<const uint4*>(block + off);
    }
#pragma unroll
    for (int o = 0; o < 2 * PC; ++o) {
      const uint32_t r[4] = {w[o].x, w[o].y, w[o].z, w[o].w};
      if (!values) {
        const int slot = (lane >> 2) + 8 * (o & 1), at = (o >> 1) * 64 + (lane & 3) * 16;
        if (at >= d || slot < u.first || slot >= u.first + u.n) continue;
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = s * value_of(r[e >> 2], e & 3);
        store_values<BF16>(x + (slot - u.first) * row_bytes + at * E, v);
      } else {
        const int at = o * 32 + (lane >> 2) * 4;
        if (at >= d) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int slot = 2 * (lane & 3) + (k & 1) + 8 * (k >> 1);
          if (slot < u.first || slot >= u.first + u.n) continue;
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = s * value_of(r[i], k);
          store_values<BF16>(x + (slot - u.first) * row_bytes + at * E, v);
        }
      }
    }
  }
}

template <bool WRITE, bool BF16, int PC>
cudaError_t launch(const StoreArgs& a, cudaStream_t stream) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  cudaLaunchConfig_t cfg = {};
  // Few blocks: a warp for each head's keys and values.  Many: as many CTAs as keep the device busy.
  const int most = (2 * a.c.heads + WARPS - 1) / WARPS, enough = (ENOUGH_CTAS * sms + a.pl.n_blocks - 1) / a.pl.n_blocks;
  cfg.gridDim = dim3((unsigned)a.pl.n_blocks, (unsigned)(most < enough ? most : enough));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return WRITE ? cudaLaunchKernelEx(&cfg, cache_write_kernel<BF16, PC>, a)
               : cudaLaunchKernelEx(&cfg, cache_read_kernel<BF16, PC>, a);
}
template <bool WRITE, bool BF16>
cudaError_t pick(const StoreArgs& a, cudaStream_t stream) {
  switch (a.c.p / 64) {
    case 1: return launch<WRITE, BF16, 1>(a, stream);
    case 2: return launch<WRITE, BF16, 2>(a, stream);
    case 3: return launch<WRITE, BF16, 3>(a, stream);
    default: return launch<WRITE, BF16, 4>(a, stream);
  }
}

}  // namespace

cudaError_t launch_cache_write(const StoreArgs& a, bool is_bf16, cudaStream_t stream) {
  return is_bf16 ? pick<true, true>(a, stream) : pick<true, false>(a, stream);
}
cudaError_t launch_cache_read(const StoreArgs& a, bool is_bf16, cudaStream_t stream) {
  return is_bf16 ? pick<false, true>(a, stream) : pick<false, false>(a, stream);
}

}  // namespace admmq
