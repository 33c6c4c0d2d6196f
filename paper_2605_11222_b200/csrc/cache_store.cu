// Rows of keys and values into the 8-bit cache, and out of it.
//
// A warp holds one block (16 tokens of a head) of keys or of values: the rows that the call adds to it, read once, are in
// registers when their largest magnitude is known, and the codes leave in the order in which the cache keeps them, 16
// bytes a lane.  Where the block is held in part, the bytes of the earlier tokens are read, rounded to the new scale if it
// has grown, and written back.
// Bound: memory for many rows (a bf16 value is read as 2 bytes and written as 1), a chain of latencies for one: position,
// page, row, maximum, store.
#include "cache.h"

namespace admmq {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr float LEAST = 9.094947017729282e-13f;     // 2^-40: magnitudes of a block that is held as zeros stay below
constexpr uint32_t MOST_BITS = 0x53800000u;         // 2^40

// N consecutive values as fp32.
template <bool BF16, int N>
__device__ __forceinline__ void load_values(const void* p, float (&v)[N]) {
  if (BF16) {
    if (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N / 8; ++i) {
        const uint4 w = ldg_stream((const char*)p + 16 * i);
        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = bf16x2_to_float2(r[e]);
          v[(8 * i + 2 * e) % N] = f.x;
          v[(8 * i + 2 * e + 1) % N] = f.y;
        }
      }
    } else {
      const uint2 w = __ldg((const uint2*)p);
      const float2 a = bf16x2_to_float2(w.x), b = bf16x2_to_float2(w.y);
      v[0] = a.x;
      v[1] = a.y;
      v[2] = b.x;
      v[3] = b.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float4 f = __ldg((const float4*)p + i);
      v[4 * i] = f.x;
      v[4 * i + 1] = f.y;
      v[4 * i + 2] = f.z;
      v[4 * i + 3] = f.w;
    }
  }
}
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

// code + 128 in the low byte.  The quotient as a division rounds it, from the reciprocal y of s: q0 = RN(x y), RN(q0 +
// (x - q0 s) y) (Markstein 1990); s is 0 (y is then 0 too, and so is x) or at least 2^-47, and |x| below 2^40, so nothing
// overflows and no remainder underflows that could decide a rounding.  Adding 1.5 * 2^23 rounds to a whole number, ties to
// even, and leaves it in the low bits.
__device__ __forceinline__ uint32_t code_of(float x, float s, float y) {
  const float q0 = __fmul_rn(x, y);
  return __float_as_uint(__fadd_rn(__fmaf_rn(__fmaf_rn(-s, q0, x), y, q0), 12583040.0f));
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

// What a warp has to do: block b of a request, of which slots [first, first + n) are rows row .. of the call.
struct Unit {
  long long index;                   // of the block for this head
  long long row;
  int first, n, head;
  bool values;
};
__device__ __forceinline__ bool find_unit(const StoreArgs& a, Unit& u) {
  const int2 job = __ldg(a.pl.blocks + blockIdx.x);
  const int which = blockIdx.y * WARPS + (threadIdx.x >> 5);
  if (which >= 2 * a.c.heads) return false;
  u.head = which >> 1;
  u.values = which & 1;
  const int row0 = __ldg(a.pl.row_start + job.x), rows = __ldg(a.pl.row_start + job.x + 1) - row0;
  const long long at = first_position(a.pl, job.x, rows, a.status);
  if (at < 0) return false;
  const int b = (int)(at / CBLOCK) + job.y, begin = max((int)at, b * CBLOCK), end = min((int)at + rows, (b + 1) * CBLOCK);
  if (begin >= end) return false;
  const long long page = block_index(a.c, a.pl, job.x, b, a.status);
  if (page < 0) return false;
  u.index = page + (long long)u.head * a.c.bpp;
  u.first = begin - b * CBLOCK;
  u.n = end - begin;
  u.row = row0 + (begin - at);
  return true;
}

// PC: the block's 64-value columns; the lane's share of them.
template <bool BF16, int PC>
__global__ void __launch_bounds__(THREADS) cache_write_kernel(const __grid_constant__ StoreArgs a) {
  Unit u;
  pdl_wait();
  if (!find_unit(a, u)) return;
  const int lane = threadIdx.x & 31, d = a.c.d;
  constexpr int E = BF16 ? 2 : 4;
  uint8_t* block = a.c.codes + u.index * a.c.block_bytes + (u.values ? 16 * a.c.p : 0);
  float* scale_at = &a.c.scale[u.index].x + (u.values ? 1 : 0);
  const float held = u.first > 0 ? *scale_at : 0.0f;
  const char* x = (const char*)(u.values ? a.v : a.k) +
                  (u.row * (u.values ? a.v_row : a.k_row) + u.head * (u.values ? a.v_head : a.k_head)) * E;
  const long long row_bytes = (u.values ? a.v_row : a.k_row) * E;

  // the lane's rows: keys [h][token half][16 values of one token], values [c][4 tokens][4 values]
  float v[2 * PC][16];
  uint32_t top = 0;
#pragma unroll
  for (int o = 0; o < 2 * PC; ++o) {
    if (!u.values) {
      const int slot = (lane >> 2) + 8 * (o & 1), at = (o >> 1) * 64 + (lane & 3) * 16;
      if (slot >= u.first && slot < u.first + u.n && at < d) {
        load_values<BF16>(x + (slot - u.first) * row_bytes + at * E, v[o]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[o][e] = 0.0f;
      }
    } else {
      const int at = o * 32 + (lane >> 2) * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int slot = 2 * (lane & 3) + (k & 1) + 8 * (k >> 1);
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        if (slot >= u.first && slot < u.first + u.n && at < d) load_values<BF16>(x + (slot - u.first) * row_bytes + at * E, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[o][4 * k + e] = f[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(v[o][e]) & 0x7fffffffu);
  }
  // (the order of the bit patterns is that of the magnitudes, with infinity and NaN on top)
  top = __reduce_max_sync(0xffffffffu, top);
  const float most = __uint_as_float(top);
  const bool bad = top >= MOST_BITS || held != held;
  const float add = most < LEAST ? 0.0f : __fmul_rn(most, 1.0f / 127.0f);
  const float s = bad ? __int_as_float(0x7fc00000) : fmaxf(held, add);
  const bool zeros = bad || s == 0.0f;
  const float y = zeros ? 0.0f : __frcp_rn(s), sc = zeros ? 0.0f : s, r = zeros ? 0.0f : __fdiv_rn(held, s);
  const bool again = u.first > 0 && !(s == held);    // earlier tokens are rounded again
  if (lane == 0) *scale_at = s;

#pragma unroll
  for (int o = 0; o < 2 * PC; ++o) {
    if (!u.values) {
      const int slot = (lane >> 2) + 8 * (o & 1), at = (o >> 1) * 64 + (lane & 3) * 16;
      uint4* dst = reinterpret_cast<uint4*>(block + (o >> 1) * 1024 + slot * 64 + (lane & 3) * 16);
      if (at >= d) continue;
      if (slot >= u.first && slot < u.first + u.n) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t k[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) k[e] = zeros ? 128u : code_of(v[o][4 * i + e], sc, y);
          w[i] = pack4(k[0], k[1], k[2], k[3]);
        }
        *dst = make_uint4(w[0], w[1], w[2], w[3]);
      } else if (slot < u.first && again) {
        const uint4 old = *dst;
        uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = pack4(rounded_again(w[i], 0, r), rounded_again(w[i], 1, r), rounded_again(w[i], 2, r), rounded_again(w[i], 3, r));
        *dst = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      const int at = o * 32 + (lane >> 2) * 4;
      uint4* dst = reinterpret_cast<uint4*>(block + o * 512 + lane * 16);
      if (at >= d) continue;
      // does the chunk hold a row of the call, or an earlier one that changes?
      const int low = 2 * (lane & 3);
      bool mine = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int slot = low + (k & 1) + 8 * (k >> 1);
        mine |= slot < u.first + u.n && (slot >= u.first || again);
      }
      if (!mine) continue;
      uint32_t w[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
      if (u.first > 0) {
        const uint4 old = *dst;
        w[0] = old.x;
        w[1] = old.y;
        w[2] = old.z;
        w[3] = old.w;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int slot = low + (k & 1) + 8 * (k >> 1);
          c[k] = w[i] >> (8 * k);
          if (slot >= u.first && slot < u.first + u.n) c[k] = zeros ? 128u : code_of(v[o][4 * k + i], sc, y);
          else if (slot < u.first && again) c[k] = rounded_again(w[i], k, r);
        }
        w[i] = pack4(c[0], c[1], c[2], c[3]);
      }
      *dst = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

template <bool BF16, int PC>
__global__ void __launch_bounds__(THREADS) cache_read_kernel(const __grid_constant__ StoreArgs a) {
  Unit u;
  pdl_wait();
  const int lane = threadIdx.x & 31, d = a.c.d;
  constexpr int E = BF16 ? 2 : 4;
  if (!find_unit(a, u)) {
    // rows of a request that takes no part, or of a page that does not exist, read as zero
    const int2 job = __ldg(a.pl.blocks + blockIdx.x);
    const int which = blockIdx.y * WARPS + (threadIdx.x >> 5);
    if (which >= 2 * a.c.heads) return;
    const int row0 = __ldg(a.pl.row_start + job.x), rows = __ldg(a.pl.row_start + job.x + 1) - row0;
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
    for (int i = begin; i < end; ++i) {
      char* p = (char*)((which & 1) ? a.v : a.k) + ((row0 + i) * ((which & 1) ? a.v_row : a.k_row) +
                                                    (which >> 1) * ((which & 1) ? a.v_head : a.k_head)) * E;
      for (int e = lane; e < d * E / 4; e += 32) reinterpret_cast<uint32_t*>(p)[e] = 0u;
    }
    return;
  }
  const uint8_t* block = a.c.codes + u.index * a.c.block_bytes + (u.values ? 16 * a.c.p : 0);
  const float s = *(&a.c.scale[u.index].x + (u.values ? 1 : 0));
  char* x = (char*)(u.values ? a.v : a.k) +
            (u.row * (u.values ? a.v_row : a.k_row) + u.head * (u.values ? a.v_head : a.k_head)) * E;
  const long long row_bytes = (u.values ? a.v_row : a.k_row) * E;
  uint4 w[2 * PC];
#pragma unroll
  for (int o = 0; o < 2 * PC; ++o) {
    const int at = u.values ? o * 32 + (lane >> 2) * 4 : (o >> 1) * 64 + (lane & 3) * 16;
    const int off = u.values ? o * 512 + lane * 16 : (o >> 1) * 1024 + ((lane >> 2) + 8 * (o & 1)) * 64 + (lane & 3) * 16;
    if (at < d) w[o] = *reinterpret_cast<const uint4*>(block + off);
  }
#pragma unroll
  for (int o = 0; o < 2 * PC; ++o) {
    const uint32_t r[4] = {w[o].x, w[o].y, w[o].z, w[o].w};
    if (!u.values) {
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

template <bool WRITE, bool BF16, int PC>
cudaError_t launch(const StoreArgs& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.pl.n_blocks, (unsigned)((2 * a.c.heads + WARPS - 1) / WARPS));
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
