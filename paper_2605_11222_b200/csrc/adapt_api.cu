// C entry points of admmq_adapt.h: argument checks and kernel selection, plus packing and the check of a bank.
#include <algorithm>
#include <atomic>

#include "../../include/admmq_testing.h"
#include "adapt.h"

namespace admmq {

extern std::atomic<long long> g_linear_wait_limit;
extern std::atomic<int> g_linear_hold_loads;

int device_sms() {
  constexpr int MAX_DEVICES = 64;
  static std::atomic<int> known[MAX_DEVICES];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

namespace {

// One thread a word: 8 codes of one output channel.
__global__ void __launch_bounds__(256)
pack_codes_kernel(const unsigned char* __restrict__ codes, int d_in, int d_out, int nib, int bits,
                  uint32_t* __restrict__ out, int* status) {
  const long long total = (long long)nib * BLOCK_WORDS * d_out;
  const int words = nib * BLOCK_WORDS;
  for (long long o = (long long)blockIdx.x * 256 + threadIdx.x; o < total; o += (long long)gridDim.x * 256) {
    const long long j = o / words;
    const int w = (int)(o - j * words), i = 8 * w;
    uint32_t v = 0u;
    if (i < d_in) {
      const uint2 c = *reinterpret_cast<const uint2*>(codes + j * d_in + i);
      uint32_t all = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t k = ((e < 4 ? c.x : c.y) >> (8 * (e & 3))) & 0xffu;
        all |= k;
        v |= (k & 15u) << (4 * ((e & 1) * 4 + (e >> 1)));
      }
      if (all >> bits) raise_status(status, ADMMQ_ERR_INVALID_ARG);
    }
    out[((long long)(w / BLOCK_WORDS) * d_out + j) * BLOCK_WORDS + w % BLOCK_WORDS] = v;
  }
}
__global__ void __launch_bounds__(256)
pack_grid_kernel(const float* __restrict__ scale, const float* __restrict__ zero, int groups, int d_out,
                 float2* __restrict__ out) {
  const long long total = (long long)groups * d_out;
  for (long long o = (long long)blockIdx.x * 256 + threadIdx.x; o < total; o += (long long)gridDim.x * 256) {
    const long long g = o / d_out, j = o - g * d_out;
    out[o] = make_float2(scale[j * groups + g], zero[j * groups + g]);
  }
}
// 8 bf16 values a thread and step; an exponent of all ones is infinity or NaN.
__global__ void __launch_bounds__(256) finite_kernel(const uint4* __restrict__ v, long long n, int* status) {
  bool bad = false;
  for (long long o = (long long)blockIdx.x * 256 + threadIdx.x; o < n; o += (long long)gridDim.x * 256) {
    const uint4 x = v[o];
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7f800000u) == 0x7f800000u || (w[e] & 0x7f80u) == 0x7f80u;
  }
  if (bad) raise_status(status, ST_NONFINITE);
}
__global__ void finite_f32_kernel(const float* __restrict__ v, int n, int* status) {
  bool bad = false;
  for (int i = threadIdx.x; i < n; i += blockDim.x) bad |= !isfinite(v[i]);
  if (bad) raise_status(status, ST_NONFINITE);
}

bool aligned(const void* p, size_t a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
unsigned grid_for(long long items) {
  const long long b = (items + 255) / 256;
  return (unsigned)(b < 1 ? 1 : b > 2368 ? 2368 : b);
}
admmq_status from(cudaError_t e) { return e == cudaSuccess ? ADMMQ_OK : ADMMQ_ERR_CUDA; }

admmq_status check_sizes(int d_in, int d_out, int group_size) {
  if (d_in < 8 || d_in > ADMMQ_MAX_D_IN || d_in % 8) return ADMMQ_ERR_SHAPE;
  if (d_out < 8 || d_out > (1 << 20) || d_out % 8) return ADMMQ_ERR_SHAPE;
  if (group_size < 0 || group_size > d_in) return ADMMQ_ERR_SHAPE;
  const int gs = group_size ? group_size : d_in;
  if (d_in % gs) return ADMMQ_ERR_SHAPE;
  return gs != d_in && gs % CODE_BLOCK ? ADMMQ_ERR_SHAPE : ADMMQ_OK;
}
admmq_status check_bank(const admmq_adapters* b) {
  if (b->struct_size != sizeof(admmq_adapters)) return ADMMQ_ERR_INVALID_ARG;
  if (!aligned(b->d_down, 16) || !aligned(b->d_up, 16) || !aligned(b->d_scale, 4)) return ADMMQ_ERR_INVALID_ARG;
  if (b->n_adapters < 1 || b->n_adapters > ADMMQ_ADAPT_MAX_ADAPTERS) return ADMMQ_ERR_SHAPE;
  return b->rank < 8 || b->rank > ADMMQ_ADAPT_MAX_RANK || b->rank % 8 ? ADMMQ_ERR_SHAPE : ADMMQ_OK;
}
bool rows_ok(long long n) { return n >= 0 && n <= ADMMQ_ADAPT_MAX_ROWS; }
bool checkpoint_ok(long long n_rows, int width) {
  return width >= 8 && width <= (1 << 20) && width % 8 == 0 && rows_ok(n_rows) &&
         n_rows * ((width + ADMMQ_CHECKPOINT_BLOCK - 1) / ADMMQ_CHECKPOINT_BLOCK) <= CHECKPOINT_MAX_BLOCKS;
}

admmq_status linear(bool grad, const admmq_packed_layer* layer, const admmq_adapters* bank, long long n_rows,
                    const int* row_adapter, const void* x, long long ldx, void* y, long long ldy, float* h,
                    int* d_status, void* cuda_stream) {
  if (!layer || layer->struct_size != sizeof(admmq_packed_layer)) return ADMMQ_ERR_INVALID_ARG;
  admmq_status st = check_sizes(layer->d_in, layer->d_out, layer->group_size);
  if (st != ADMMQ_OK) return st;
  if (!aligned(layer->d_packed, 16) || !aligned(layer->d_grid, 16) || !aligned(d_status, 4)) return ADMMQ_ERR_INVALID_ARG;
  if (bank && (st = check_bank(bank)) != ADMMQ_OK) return st;
  if (!rows_ok(n_rows)) return ADMMQ_ERR_SHAPE;
  const int K = grad ? layer->d_out : layer->d_in, M = grad ? layer->d_in : layer->d_out;
  if (ldx < K || ldx % 8 || ldy < M || ldy % 8) return ADMMQ_ERR_SHAPE;
  if (n_rows == 0) return ADMMQ_OK;
  if (!aligned(x, 16) || !aligned(y, 16)) return ADMMQ_ERR_INVALID_ARG;
  if (bank && (!aligned(row_adapter, 4) || !aligned(h, 16))) return ADMMQ_ERR_INVALID_ARG;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const int gs = layer->group_size ? layer->group_size : layer->d_in;
  const PackedLayer L = {(const uint32_t*)layer->d_packed, (const float2*)layer->d_grid, layer->d_in, layer->d_out,
                         (layer->d_in + CODE_BLOCK - 1) / CODE_BLOCK, gs};
  AdapterView ad = {};
  if (bank) {
    ad = {(const bf16*)(grad ? bank->d_up : bank->d_down), (const bf16*)(grad ? bank->d_down : bank->d_up),
          bank->d_scale, bank->n_adapters, bank->rank};
    // multiprocessors that the projection leaves to the contraction, which it overlaps
    const int sms = device_sms();
    if (sms <= 0) return ADMMQ_ERR_CUDA;
    const bool small = !grad && n_rows <= SMALL_ROWS;
    const int spare = small ? 0 : (int)std::max(0LL, sms - plan_linear_tc(grad, L, n_rows, sms).ctas);
    const cudaError_t e = launch_shrink((const bf16*)x, ldx, n_rows, K, ad, row_adapter, h, spare, d_status, stream);
    if (e != cudaSuccess) return ADMMQ_ERR_CUDA;
  }
  if (!grad && n_rows <= SMALL_ROWS)
    return from(launch_linear_small(L, bank ? &ad : nullptr, (int)n_rows, row_adapter, (const bf16*)x, ldx, (bf16*)y,
                                    ldy, h, stream));
  return from(launch_linear_tc(grad, L, bank ? &ad : nullptr, n_rows, row_adapter, (const bf16*)x, ldx, (bf16*)y, ldy,
                               h, d_status, stream));
}

admmq_status check_qk(const admmq_qk_args* a, bool backward) {
  if (!a || a->struct_size != sizeof(admmq_qk_args)) return ADMMQ_ERR_INVALID_ARG;
  if (a->dtype != ADMMQ_F32 && a->dtype != ADMMQ_BF16) return ADMMQ_ERR_INVALID_ARG;
  if (a->q_heads < 1 || a->k_heads < 0 || a->q_heads > 65536 || a->k_heads > 65536) return ADMMQ_ERR_SHAPE;
  if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16) return ADMMQ_ERR_SHAPE;
  if (a->rot_dim < 16 || a->rot_dim > a->head_dim || a->rot_dim % 16) return ADMMQ_ERR_SHAPE;
  if (!rows_ok(a->n_rows) || a->n_positions < 1) return ADMMQ_ERR_SHAPE;
  if (!(a->eps >= 0.0)) return ADMMQ_ERR_INVALID_ARG;
  const int e = a->dtype == ADMMQ_BF16 ? 8 : 4;
  const bool k = a->k_heads > 0;
  if (a->q_row % e || a->q_head % e || a->out_q_row % e || a->out_q_head % e) return ADMMQ_ERR_SHAPE;
  if (k && (a->k_row % e || a->k_head % e || a->out_k_row % e || a->out_k_head % e)) return ADMMQ_ERR_SHAPE;
  if (!aligned(a->d_wq, 16) || (k && !aligned(a->d_wk, 16))) return ADMMQ_ERR_INVALID_ARG;
  if (!aligned(a->d_cos, 16) || !aligned(a->d_sin, 16) || !aligned(a->d_status, 4)) return ADMMQ_ERR_INVALID_ARG;
  if (a->n_rows > 0) {
    if (!aligned(a->d_q, 16) || !aligned(a->d_out_q, 16) || !aligned(a->d_pos, 4)) return ADMMQ_ERR_INVALID_ARG;
    if (k && (!aligned(a->d_k, 16) || !aligned(a->d_out_k, 16))) return ADMMQ_ERR_INVALID_ARG;
  }
  if (backward) {
    if (a->dy_q_row % e || a->dy_q_head % e || (k && (a->dy_k_row % e || a->dy_k_head % e))) return ADMMQ_ERR_SHAPE;
    if (a->n_rows > 0 && (!aligned(a->d_dy_q, 16) || (k && !aligned(a->d_dy_k, 16)))) return ADMMQ_ERR_INVALID_ARG;
    if (!aligned(a->d_grad_wq, 4) || (k && !aligned(a->d_grad_wk, 4))) return ADMMQ_ERR_INVALID_ARG;
    if (!aligned(a->d_workspace, 16)) return ADMMQ_ERR_INVALID_ARG;
    if (a->workspace_bytes < admmq_qk_workspace_bytes(a->head_dim)) return ADMMQ_ERR_WORKSPACE;
  }
  return ADMMQ_OK;
}

}  // namespace
}  // namespace admmq

using namespace admmq;

extern "C" {

size_t admmq_packed_bytes(int d_in, int d_out) {
  if (check_sizes(d_in, d_out, 0) != ADMMQ_OK) return 0;
  return (size_t)((d_in + CODE_BLOCK - 1) / CODE_BLOCK) * d_out * (CODE_BLOCK / 2);
}
size_t admmq_grid_bytes(int d_in, int d_out, int group_size) {
  if (check_sizes(d_in, d_out, group_size) != ADMMQ_OK) return 0;
  return (size_t)(group_size ? d_in / group_size : 1) * d_out * sizeof(float2);
}

admmq_status admmq_pack_layer(const unsigned char* d_codes, const float* d_scale, const float* d_zero, int d_in,
                              int d_out, int bits, int group_size, void* d_packed, void* d_grid, int* d_status,
                              void* cuda_stream) {
  if (bits < 2 || bits > ADMMQ_MAX_BITS) return ADMMQ_ERR_SHAPE;
  if (bits > ADMMQ_ADAPT_MAX_BITS) return ADMMQ_ERR_UNSUPPORTED;
  const admmq_status st = check_sizes(d_in, d_out, group_size);
  if (st != ADMMQ_OK) return st;
  if (!aligned(d_codes, 16) || !aligned(d_scale, 4) || !aligned(d_zero, 4) || !aligned(d_packed, 16) ||
      !aligned(d_grid, 16) || !aligned(d_status, 4))
    return ADMMQ_ERR_INVALID_ARG;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const int nib = (d_in + CODE_BLOCK - 1) / CODE_BLOCK, groups = group_size ? d_in / group_size : 1;
  pack_codes_kernel<<<grid_for((long long)nib * BLOCK_WORDS * d_out), 256, 0, stream>>>(d_codes, d_in, d_out, nib, bits,
                                                                                     (uint32_t*)d_packed, d_status);
  pack_grid_kernel<<<grid_for((long long)groups * d_out), 256, 0, stream>>>(d_scale, d_zero, groups, d_out,
                                                                         (float2*)d_grid);
  return from(cudaGetLastError());
}

admmq_status admmq_adapters_check(const admmq_adapters* bank, int d_in, int d_out, int* d_status, void* cuda_stream) {
  if (!bank) return ADMMQ_ERR_INVALID_ARG;
  admmq_status st = check_sizes(d_in, d_out, 0);
  if (st == ADMMQ_OK) st = check_bank(bank);
  if (st != ADMMQ_OK) return st;
  if (!aligned(d_status, 4)) return ADMMQ_ERR_INVALID_ARG;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const long long rows = (long long)bank->n_adapters * bank->rank;
  finite_kernel<<<grid_for(rows * d_in / 8), 256, 0, stream>>>((const uint4*)bank->d_down, rows * d_in / 8, d_status);
  finite_kernel<<<grid_for(rows * d_out / 8), 256, 0, stream>>>((const uint4*)bank->d_up, rows * d_out / 8, d_status);
  finite_f32_kernel<<<1, 256, 0, stream>>>(bank->d_scale, bank->n_adapters, d_status);
  return from(cudaGetLastError());
}

admmq_status admmq_linear_forward(const admmq_packed_layer* layer, const admmq_adapters* bank, long long n_rows,
                                  const int* d_row_adapter, const void* d_x, long long ldx, void* d_y, long long ldy,
                                  float* d_h, int* d_status, void* cuda_stream) {
  return linear(false, layer, bank, n_rows, d_row_adapter, d_x, ldx, d_y, ldy, d_h, d_status, cuda_stream);
}
admmq_status admmq_linear_grad_input(const admmq_packed_layer* layer, const admmq_adapters* bank, long long n_rows,
                                     const int* d_row_adapter, const void* d_dy, long long lddy, void* d_dx,
                                     long long lddx, float* d_u, int* d_status, void* cuda_stream) {
  return linear(true, layer, bank, n_rows, d_row_adapter, d_dy, lddy, d_dx, lddx, d_u, d_status, cuda_stream);
}

admmq_status admmq_adapter_grad(const admmq_adapter_grad_args* a, void* cuda_stream) {
  if (!a || a->struct_size != sizeof(admmq_adapter_grad_args)) return ADMMQ_ERR_INVALID_ARG;
  const admmq_status st = check_sizes(a->d_in, a->d_out, 0);
  if (st != ADMMQ_OK) return st;
  if (a->n_adapters < 1 || a->n_adapters > ADMMQ_ADAPT_MAX_ADAPTERS) return ADMMQ_ERR_SHAPE;
  if (a->rank < 8 || a->rank > ADMMQ_ADAPT_MAX_RANK || a->rank % 8) return ADMMQ_ERR_SHAPE;
  if (!rows_ok(a->n_rows)) return ADMMQ_ERR_SHAPE;
  if (!aligned(a->d_offsets, 4) || !aligned(a->d_grad_down, 16) || !aligned(a->d_grad_up, 16)) return ADMMQ_ERR_INVALID_ARG;
  if (a->n_rows > 0) {
    if (a->d_x ? (a->ldx < a->d_in || a->ldx % 8) : false) return ADMMQ_ERR_SHAPE;
    if (a->lddy < a->d_out || a->lddy % 8) return ADMMQ_ERR_SHAPE;
    if (!aligned(a->d_order, 4) || !aligned(a->d_h, 16) || !aligned(a->d_u, 16) || !aligned(a->d_dy, 16))
      return ADMMQ_ERR_INVALID_ARG;
    if (a->d_x ? !aligned(a->d_x, 16) : !aligned(a->d_x_codes, 16) || !aligned(a->d_x_scale, 4)) return ADMMQ_ERR_INVALID_ARG;
  }
  return from(launch_adapter_grad(*a, (cudaStream_t)cuda_stream));
}

admmq_status admmq_checkpoint_save(const void* d_x, admmq_dtype dtype, long long n_rows, int width, long long ldx,
                                   signed char* d_codes, float* d_scale, void* cuda_stream) {
  if (dtype != ADMMQ_F32 && dtype != ADMMQ_BF16) return ADMMQ_ERR_INVALID_ARG;
  if (!checkpoint_ok(n_rows, width)) return ADMMQ_ERR_SHAPE;
  if (ldx < width || ldx % (dtype == ADMMQ_BF16 ? 8 : 4)) return ADMMQ_ERR_SHAPE;
  if (n_rows == 0) return ADMMQ_OK;
  if (!aligned(d_x, 16) || !aligned(d_codes, 16) || !aligned(d_scale, 4)) return ADMMQ_ERR_INVALID_ARG;
  return from(launch_checkpoint_save(d_x, dtype == ADMMQ_BF16, n_rows, width, ldx, (int8_t*)d_codes, d_scale,
                                     (cudaStream_t)cuda_stream));
}
admmq_status admmq_checkpoint_restore(const signed char* d_codes, const float* d_scale, long long n_rows, int width,
                                      void* d_out, admmq_dtype dtype, long long ldo, void* cuda_stream) {
  if (dtype != ADMMQ_F32 && dtype != ADMMQ_BF16) return ADMMQ_ERR_INVALID_ARG;
  if (!checkpoint_ok(n_rows, width)) return ADMMQ_ERR_SHAPE;
  if (ldo < width || ldo % (dtype == ADMMQ_BF16 ? 8 : 4)) return ADMMQ_ERR_SHAPE;
  if (n_rows == 0) return ADMMQ_OK;
  if (!aligned(d_out, 16) || !aligned(d_codes, 16) || !aligned(d_scale, 4)) return ADMMQ_ERR_INVALID_ARG;
  return from(launch_checkpoint_restore((const int8_t*)d_codes, d_scale, n_rows, width, d_out, dtype == ADMMQ_BF16,
                                        ldo, (cudaStream_t)cuda_stream));
}

size_t admmq_qk_workspace_bytes(int head_dim) {
  if (head_dim < 16 || head_dim > 256 || head_dim % 16) return 0;
  return (size_t)2 * QK_GRAD_BLOCKS * head_dim * sizeof(float);
}
admmq_status admmq_qk_norm_rope(const admmq_qk_args* args, void* cuda_stream) {
  const admmq_status st = check_qk(args, false);
  if (st != ADMMQ_OK) return st;
  if (args->n_rows == 0) return ADMMQ_OK;
  return from(launch_qk(*args, false, (cudaStream_t)cuda_stream));
}
admmq_status admmq_qk_norm_rope_backward(const admmq_qk_args* args, void* cuda_stream) {
  const admmq_status st = check_qk(args, true);
  if (st != ADMMQ_OK) return st;
  return from(launch_qk(*args, true, (cudaStream_t)cuda_stream));
}

admmq_status admmq_test_linear_set_wait(long long wait_limit_cycles, int hold_loads) {
  if (wait_limit_cycles < 1000) return ADMMQ_ERR_INVALID_ARG;
  g_linear_wait_limit.store(wait_limit_cycles, std::memory_order_relaxed);
  g_linear_hold_loads.store(hold_loads ? 1 : 0, std::memory_order_relaxed);
  return ADMMQ_OK;
}

}  // extern "C"
