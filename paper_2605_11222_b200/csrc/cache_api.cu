// C entry points of admmq_cache.h: argument checks, the index of a call's rows, kernel selection.
#include <algorithm>

#include "cache.h"

namespace admmq {
namespace {

constexpr int MAX_HEADS = 4096;
constexpr long long MAX_POSITIONS = 1LL << 30;
// Packed rows of a request up to which they are a few (sixteen at a time, each reading the cache through the L2 cache again):
// 64, or 128 where the call has no more in all.  32 query and 8 key heads of 128, measured, us, few against many:
// one request over 500 tokens 64 rows 11, 23, 128 rows 19, 24, 256 rows 25, 25; over 4000 17, 35, 27, 35, 42, 36; eight
// requests over 4000 64 rows 69, 64, 128 rows 116, 66.
constexpr int MOST_FEW = 64, MOST_FEW_ALONE = 128;

bool aligned(const void* p, size_t a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
admmq_status from(cudaError_t e) { return e == cudaSuccess ? ADMMQ_OK : ADMMQ_ERR_CUDA; }
int log2_of(int n) {
  int s = 0;
  while ((1 << s) < n) ++s;
  return s;
}
// Whether the rows and heads of an output lie apart (the stride of a single one does not matter).
bool apart(long long rows, long long row, int heads, long long head, int d) {
  if (rows < 2) return heads < 2 || head >= d;
  if (heads < 2) return row >= d;
  return row >= head ? head >= d && row >= (heads - 1) * head + d : row >= d && head >= (rows - 1) * row + d;
}
admmq_status check_sizes(int n_pages, int kv_heads, int head_dim, int page_size) {
  if (n_pages < 1 || kv_heads < 1 || kv_heads > MAX_HEADS) return ADMMQ_ERR_SHAPE;
  if (head_dim < 16 || head_dim > ADMMQ_CACHE_MAX_HEAD || head_dim % 16) return ADMMQ_ERR_SHAPE;
  if (page_size < CBLOCK || page_size > ADMMQ_CACHE_MAX_PAGE || page_size & (page_size - 1)) return ADMMQ_ERR_SHAPE;
  // (blocks are counted in 32 bits; so many do not fit a device)
  return (long long)n_pages * kv_heads * (page_size / CBLOCK) > 0x7fffffffLL ? ADMMQ_ERR_SHAPE : ADMMQ_OK;
}
admmq_status view_cache(const admmq_cache* c, CacheView* v) {
  if (!c || c->struct_size != sizeof(admmq_cache)) return ADMMQ_ERR_INVALID_ARG;
  const admmq_status st = check_sizes(c->n_pages, c->kv_heads, c->head_dim, c->page_size);
  if (st != ADMMQ_OK) return st;
  if (!aligned(c->d_codes, 16) || !aligned(c->d_scale, 16)) return ADMMQ_ERR_INVALID_ARG;
  const int p = (c->head_dim + 63) / 64 * 64;
  *v = {(uint8_t*)c->d_codes, (float2*)c->d_scale, c->n_pages, c->kv_heads, c->head_dim, p,
        c->page_size / CBLOCK, log2_of(c->page_size / CBLOCK), 2 * CBLOCK * p};
  return ADMMQ_OK;
}

// Blocks that `rows` rows touch at most, tiles of packed rows.
long long blocks_of(long long rows) { return rows > 0 ? (rows + 2 * CBLOCK - 2) / CBLOCK : 0; }
long long tiles_of(long long packed, int rows) { return (packed + rows - 1) / rows; }
bool is_few(long long packed, long long all) { return packed <= MOST_FEW || all <= MOST_FEW_ALONE; }
long long round4(long long n) { return (n + 3) & ~3LL; }
// The index of a call's rows: the first row of every request and their number (for the caller; the kernels find it in the
// entries below), then an entry of four for every block that rows may touch and for every tile.
struct IndexSizes {
  long long rows, blocks, small, big, small_rows;   // small_rows: most packed rows that a small tile holds
  long long ints(int n) const { return round4(n + 1) + 4 * (blocks + small + big); }
};
bool index_sizes(const long long* lengths, int n, int group, IndexSizes* s) {
  *s = {};
  if (!lengths || n < 1 || n > (1 << 24) || group < 1 || group > 1024) return false;
  for (int i = 0; i < n; ++i) {
    if (lengths[i] < 0 || lengths[i] > MAX_POSITIONS) return false;
    s->rows += lengths[i];
    if (s->rows * group > MAX_POSITIONS) return false;
    s->blocks += blocks_of(lengths[i]);
  }
  for (int i = 0; i < n; ++i) {
    const long long packed = lengths[i] * group;
    if (is_few(packed, s->rows * group)) s->small_rows = std::max(s->small_rows, std::min(packed, (long long)FEW_ROWS));
    (is_few(packed, s->rows * group) ? s->small : s->big) += tiles_of(packed, is_few(packed, s->rows * group) ? FEW_ROWS : MANY_ROWS);
  }
  return s->ints(n) <= 0x7fffffffLL;
}
admmq_status view_plan(const admmq_cache_plan* p, const CacheView& c, PlanView* v) {
  if (!p || p->struct_size != sizeof(admmq_cache_plan)) return ADMMQ_ERR_INVALID_ARG;
  if (p->n_requests < 1 || p->max_pages < 1 || p->group < 1 || p->n_rows < 0 || p->n_blocks < 0 || p->n_small < 0 || p->n_big < 0 ||
      p->small_rows < 0 || p->small_rows > FEW_ROWS)
    return ADMMQ_ERR_SHAPE;
  const long long capacity = (long long)p->max_pages * c.bpp * CBLOCK;
  if (capacity > MAX_POSITIONS || p->n_rows > MAX_POSITIONS) return ADMMQ_ERR_SHAPE;
  if (!aligned(p->d_tables, 4) || !aligned(p->d_held, 4) || !aligned(p->d_index, 16)) return ADMMQ_ERR_INVALID_ARG;
  const int* at = p->d_index + round4(p->n_requests + 1);
  const int* tiles = at + 4LL * p->n_blocks;
  *v = {p->d_tables, p->d_held, (const int4*)at, (const int4*)tiles, (const int4*)tiles + p->n_small,
        p->max_pages, p->group, p->n_blocks, p->n_small, p->n_big, p->small_rows, capacity};
  return ADMMQ_OK;
}

admmq_status store(bool write, const admmq_cache* cache, const admmq_cache_plan* plan, admmq_dtype dtype, const void* k,
                   long long k_row, long long k_head, const void* v, long long v_row, long long v_head, int* d_status,
                   void* cuda_stream) {
  StoreArgs a = {};
  admmq_status st = view_cache(cache, &a.c);
  if (st == ADMMQ_OK) st = view_plan(plan, a.c, &a.pl);
  if (st != ADMMQ_OK) return st;
  if (dtype != ADMMQ_F32 && dtype != ADMMQ_BF16) return ADMMQ_ERR_INVALID_ARG;
  const int e = dtype == ADMMQ_BF16 ? 8 : 4;
  if (k_row % e || k_head % e || v_row % e || v_head % e) return ADMMQ_ERR_SHAPE;
  if (!write && !(apart(plan->n_rows, k_row, a.c.heads, k_head, a.c.d) && apart(plan->n_rows, v_row, a.c.heads, v_head, a.c.d)))
    return ADMMQ_ERR_SHAPE;
  if (!aligned(d_status, 4)) return ADMMQ_ERR_INVALID_ARG;
  if (plan->n_rows == 0) return ADMMQ_OK;
  if (!aligned(k, 16) || !aligned(v, 16)) return ADMMQ_ERR_INVALID_ARG;
  a.k = k;
  a.v = v;
  a.k_row = k_row;
  a.k_head = k_head;
  a.v_row = v_row;
  a.v_head = v_head;
  a.status = d_status;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  return from(write ? launch_cache_write(a, dtype == ADMMQ_BF16, stream) : launch_cache_read(a, dtype == ADMMQ_BF16, stream));
}

// Workspace of one kind of tiles: for every CTA what is to be joined, and two partial results.
size_t part_bytes(const CacheView& c, bool many, int sms) {
  const size_t ctas = attend_ctas(c.p, many, sms), rows = many ? many_rows(c.p) : FEW_ROWS;
  return ctas * (sizeof(Join) + 2 * rows * (c.p * sizeof(float) + sizeof(float2)));
}
size_t workspace_of(const CacheView& c, const PlanView& p, int sms) {
  return (p.n_small ? part_bytes(c, false, sms) : 0) + (p.n_big ? part_bytes(c, true, sms) : 0);
}

}  // namespace
}  // namespace admmq

using namespace admmq;

extern "C" {

size_t admmq_cache_code_bytes(int n_pages, int kv_heads, int head_dim, int page_size) {
  if (check_sizes(n_pages, kv_heads, head_dim, page_size) != ADMMQ_OK) return 0;
  return (size_t)n_pages * kv_heads * page_size * 2 * ((head_dim + 63) / 64 * 64);
}
size_t admmq_cache_scale_bytes(int n_pages, int kv_heads, int head_dim, int page_size) {
  if (check_sizes(n_pages, kv_heads, head_dim, page_size) != ADMMQ_OK) return 0;
  return (size_t)n_pages * kv_heads * (page_size / CBLOCK) * sizeof(float2);
}

long long admmq_cache_plan_ints(const long long* lengths, int n_requests, int group) {
  IndexSizes s;
  return index_sizes(lengths, n_requests, group, &s) ? s.ints(n_requests) : -1;
}
admmq_status admmq_cache_plan_fill(const long long* lengths, int n_requests, int group, int* index, admmq_cache_plan* plan) {
  IndexSizes s;
  if (!index || !plan || plan->struct_size != sizeof(admmq_cache_plan)) return ADMMQ_ERR_INVALID_ARG;
  if (!index_sizes(lengths, n_requests, group, &s)) return ADMMQ_ERR_SHAPE;
  int* blocks = index + round4(n_requests + 1);
  int* small = blocks + 4 * s.blocks;
  int* big = small + 4 * s.small;
  for (int* p = index; p < big + 4 * s.big; ++p) *p = 0;
  int row = 0;
  for (int i = 0; i < n_requests; ++i) {
    const int rows = (int)lengths[i];
    index[i] = row;
    for (int b = 0; b < blocks_of(rows); ++b) {
      *blocks++ = i;
      *blocks++ = b;
      *blocks++ = row;
      *blocks++ = rows;
    }
    const bool few = is_few((long long)rows * group, s.rows * group);
    const int step = few ? FEW_ROWS : MANY_ROWS;
    for (long long r = 0; r < (long long)rows * group; r += step) {
      int*& t = few ? small : big;
      *t++ = i;
      *t++ = (int)r;
      *t++ = row;
      *t++ = rows;
    }
    row += rows;
  }
  index[n_requests] = row;
  plan->n_requests = n_requests;
  plan->group = group;
  plan->n_rows = s.rows;
  plan->n_blocks = (int)s.blocks;
  plan->n_small = (int)s.small;
  plan->n_big = (int)s.big;
  plan->small_rows = (int)s.small_rows;
  return ADMMQ_OK;
}

admmq_status admmq_cache_write(const admmq_cache* cache, const admmq_cache_plan* plan, admmq_dtype dtype, const void* d_k,
                               long long k_row, long long k_head, const void* d_v, long long v_row, long long v_head,
                               int* d_status, void* cuda_stream) {
  return store(true, cache, plan, dtype, d_k, k_row, k_head, d_v, v_row, v_head, d_status, cuda_stream);
}
admmq_status admmq_cache_read(const admmq_cache* cache, const admmq_cache_plan* plan, admmq_dtype dtype, void* d_k,
                              long long k_row, long long k_head, void* d_v, long long v_row, long long v_head, int* d_status,
                              void* cuda_stream) {
  return store(false, cache, plan, dtype, d_k, k_row, k_head, d_v, v_row, v_head, d_status, cuda_stream);
}

size_t admmq_cache_attend_workspace(const admmq_cache* cache, const admmq_cache_plan* plan) {
  CacheView c;
  PlanView p;
  if (view_cache(cache, &c) != ADMMQ_OK || view_plan(plan, c, &p) != ADMMQ_OK) return 0;
  const int sms = device_sms();
  return sms > 0 ? workspace_of(c, p, sms) : 0;
}
admmq_status admmq_cache_attend(const admmq_cache* cache, const admmq_cache_plan* plan, double scale, int window,
                                const void* d_q, long long q_row, long long q_head, void* d_out, long long out_row,
                                long long out_head, float* d_lse, void* d_workspace, size_t workspace_bytes, int* d_status,
                                void* cuda_stream) {
  AttendArgs a = {};
  admmq_status st = view_cache(cache, &a.c);
  if (st == ADMMQ_OK) st = view_plan(plan, a.c, &a.pl);
  if (st != ADMMQ_OK) return st;
  if (!(scale > 0.0) || scale > 1e30 || window < 0) return ADMMQ_ERR_INVALID_ARG;
  if ((long long)a.c.heads * a.pl.group > 65536) return ADMMQ_ERR_SHAPE;
  if (q_row % 8 || q_head % 8 || out_row % 8 || out_head % 8) return ADMMQ_ERR_SHAPE;
  if (!apart(plan->n_rows, out_row, a.c.heads * a.pl.group, out_head, a.c.d)) return ADMMQ_ERR_SHAPE;
  if (!aligned(d_status, 4)) return ADMMQ_ERR_INVALID_ARG;
  if (plan->n_rows == 0) return ADMMQ_OK;
  if (!aligned(d_q, 16) || !aligned(d_out, 16) || (d_lse && !aligned(d_lse, 4)) || !aligned(d_workspace, 16)) return ADMMQ_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms <= 0) return ADMMQ_ERR_CUDA;
  if (workspace_bytes < workspace_of(a.c, a.pl, sms)) return ADMMQ_ERR_WORKSPACE;
  a.q = (const bf16*)d_q;
  a.out = (bf16*)d_out;
  a.lse = d_lse;
  a.q_row = q_row;
  a.q_head = q_head;
  a.out_row = out_row;
  a.out_head = out_head;
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.window = window < MAX_POSITIONS ? window : 0;    // (positions end below)
  a.status = d_status;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  char* at = (char*)d_workspace;
  for (int many = 0; many < 2; ++many) {
    if (!(many ? a.pl.n_big : a.pl.n_small)) continue;
    const size_t ctas = attend_ctas(a.c.p, many, sms), rows = many ? many_rows(a.c.p) : FEW_ROWS;
    // (halves of the plan's tiles may be without rows: nobody begins those)
    a.by_piece = !(many && rows < MANY_ROWS) && pieces_of(a, many) <= (long long)ctas;
    a.joins = (Join*)at;
    a.part = (float*)(a.joins + ctas);
    a.part_ml = (float2*)(a.part + ctas * 2 * rows * a.c.p);
    at += part_bytes(a.c, many, sms);
    const cudaError_t e = many ? launch_cache_attend_many(a, stream) : launch_cache_attend_few(a, stream);
    if (e != cudaSuccess) return ADMMQ_ERR_CUDA;
  }
  return ADMMQ_OK;
}

}  // extern "C"
