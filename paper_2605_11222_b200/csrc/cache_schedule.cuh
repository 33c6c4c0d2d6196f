// How the kernels that attend over the cache share out their work, and how partial results are joined.
//
// Work is counted in units of a fixed number of positions.  A tile of packed rows of one request has, for every key head,
// the units that its rows see; all of them, tile after tile and head after head, are one line of T units, of which CTA c of
// G takes [c T / G, (c + 1) T / G): every CTA has the same to do, however long the requests are, and the device finds its
// part from the lengths when it runs.  A (tile, head) counts `EXTRA` units more than it has, ahead of them, for what a piece
// costs whatever its length.  A piece is what a CTA has of one (tile, head).  Pieces that are whole write the
// result; of others the CTA leaves the unnormalised sum, the maximum and the sum of weights (slot 1 where it begins the
// (tile, head), slot 0 where it goes on with one), and the join kernel adds them up in the order of the CTAs.
#pragma once
#include "cache.h"
#include "tc_ptx.cuh"

namespace admmq {

// Bounded wait of a whole warp with one answer for all its lanes.  (Inlined: setmaxnreg asks for a kernel without calls.)
struct WarpWait {
  volatile int* abort_flag;
  int* status;
  long long limit;
  __device__ __forceinline__ bool all(uint32_t bar, uint32_t parity) const {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status, limit)) != 0;
  }
};

// (Numbers below 2^32, which these nearly always are, divide in a fraction of the time.)
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
// Positions that the rows of a tile see: [lo, hi); hi = 0 where the request takes no part.
struct Span {
  int at;                              // position of the request's first row, -1: none
  int lo, hi;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, const int4& tile, int tile_rows) {
  Span s = {-1, 0, 0};
  const long long at = first_position(a.pl, tile.x, tile.w, a.status);
  if (at < 0) return s;
  const int first = tile.y / a.pl.group, last = (min(tile.y + tile_rows, tile.w * a.pl.group) - 1) / a.pl.group;
  s.at = (int)at;
  s.hi = s.at + last + 1;
  s.lo = a.window > 0 ? max(0, s.at + first - a.window + 1) : 0;
  return s;
}
// Its units: one where the request takes no part (the rows are written all the same), none for a tile without rows (a half
// of one that the request does not fill).
template <int UNIT>
__device__ __forceinline__ int units_of(const Span& s, const int4& tile, int group) {
  if (tile.y >= tile.w * group) return 0;
  return s.hi > 0 ? (s.hi + UNIT - 1) / UNIT - s.lo / UNIT : 1;
}
template <int UNIT>
__device__ __forceinline__ int units_of(const AttendArgs& a, const int4& tile, int tile_rows) {
  return units_of<UNIT>(span_of(a, tile, tile_rows), tile, a.pl.group);
}

// job(t): tile t, as the plan's tiles.  Prefix sums of the tiles' units by segments of tiles, one segment a thread.
template <int THREADS>
struct Schedule {
  long long sums[THREADS + 1];
  long long warp_sums[THREADS / 32];
  int per;
};
// All threads; returns the length of the line (of one head).
template <int UNIT, int EXTRA>
__device__ __forceinline__ int cost_of(int units) {
  return units > 0 ? units + EXTRA : 0;
}
template <int THREADS, int UNIT, int ROWS, int EXTRA, class Job>
__device__ __forceinline__ long long make_schedule(const AttendArgs& a, const Job& job, int n, Schedule<THREADS>& s) {
  const int per = (n + THREADS - 1) / THREADS, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  long long mine = 0;
  for (int t = tid * per; t < min(n, (tid + 1) * per); ++t) mine += cost_of<UNIT, EXTRA>(units_of<UNIT>(a, job(t), ROWS));
  long long run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += up;
  }
  if (lane == 31) s.warp_sums[warp] = run;
  if (tid == 0) s.per = per;
  __syncthreads();
  long long base = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) base += w < warp ? s.warp_sums[w] : 0;
  s.sums[tid] = base + run - mine;
  if (tid == THREADS - 1) s.sums[THREADS] = base + run;
  __syncthreads();
  return s.sums[THREADS];
}
// The piece that holds unit u of the line.
struct Piece {
  int tile, head;
  int4 job;
  Span span;
  long long begin, end;                // the (tile, head)'s units in the line (u may be before: of the extra ones)
};
// .. of those in segment `seg`.
template <int THREADS, int UNIT, int ROWS, int EXTRA, class Job>
__device__ __forceinline__ Piece piece_of(const AttendArgs& a, const Job& job, int n, const Schedule<THREADS>& s, int seg, long long u) {
  const int heads = a.c.heads;
  long long at = s.sums[seg] * heads;
  Piece p;
  int t = seg * s.per;
  for (;; ++t) {
    p.job = job(t);
    p.span = span_of(a, p.job, ROWS);
    const long long cost = cost_of<UNIT, EXTRA>(units_of<UNIT>(p.span, p.job, a.pl.group));
    // (It is found within the segment.  Should somebody write into `held` meanwhile, the last tile ends the search.)
    if (u < at + cost * heads || t + 1 >= n) {
      p.head = cost > 0 ? (int)min(quotient(u - at, cost), (long long)heads - 1) : 0;
      p.begin = at + p.head * cost + EXTRA;
      p.end = at + (p.head + 1) * cost;
      break;
    }
    at += cost * heads;
  }
  p.tile = t;
  return p;
}
template <int THREADS, int UNIT, int ROWS, int EXTRA, class Job>
__device__ __forceinline__ Piece find_piece(const AttendArgs& a, const Job& job, int n, const Schedule<THREADS>& s, long long u) {
  int lo = 0, hi = THREADS;            // segment: the last one with sums * heads <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (s.sums[mid] * a.c.heads <= u) lo = mid;
    else hi = mid;
  }
  return piece_of<THREADS, UNIT, ROWS, EXTRA>(a, job, n, s, lo, u);
}
// The piece after `p`; an empty one at its end where there is none.
template <int UNIT, int ROWS, int EXTRA, class Job>
__device__ __forceinline__ Piece piece_after(const AttendArgs& a, const Job& job, int n, Piece p) {
  long long cost = p.end - p.begin + EXTRA;
  if (++p.head == a.c.heads) {
    p.head = 0;
    for (cost = 0; cost == 0 && ++p.tile < n;) {
      p.job = job(p.tile);
      p.span = span_of(a, p.job, ROWS);
      cost = cost_of<UNIT, EXTRA>(units_of<UNIT>(p.span, p.job, a.pl.group));
    }
  }
  p.begin = cost > 0 ? p.end + EXTRA : p.end;
  p.end += cost;
  return p;
}
// CTAs that get work: at least `least` units each.
__device__ __forceinline__ int active_ctas(long long total, int least) {
  const long long most = quotient(total + least - 1, least);
  return (int)(most < (long long)gridDim.x ? most : (long long)gridDim.x);
}
// CTA c has [line_at(c), line_at(c + 1)): total / ctas units, and one more the first total % ctas.
__device__ __forceinline__ long long line_at(long long total, int c, int ctas) {
  const long long each = quotient(total, ctas), more = total - each * ctas;
  return c * each + min((long long)c, more);
}
// What is to be joined of a (tile, head), told by the CTA that begins it.
__device__ __forceinline__ void tell_join(const AttendArgs& a, const Piece& p, int tile_rows, int first, int last) {
  const Join j = {first, last, p.head, p.job.y, p.job.z, min(tile_rows, p.job.w * a.pl.group - p.job.y), {0, 0}};
  if (a.by_piece) a.joins[p.tile * a.c.heads + p.head] = j;
  else if (last > first) a.joins[first] = j;
}
// And, where joins go by CTA, by one that begins none which others end.
__device__ __forceinline__ void tell_none(const AttendArgs& a, int cta) {
  if (!a.by_piece) a.joins[cta] = {cta, cta, 0, 0, 0, 0, {0, 0}};
}
// The CTA that has unit u.
__device__ __forceinline__ int cta_of(long long u, long long total, int ctas) {
  const long long each = quotient(total, ctas), more = total - each * ctas, long_ones = more * (each + 1);
  return (int)(u < long_ones ? quotient(u, each + 1) : more + quotient(u - long_ones, each));
}

}  // namespace admmq
