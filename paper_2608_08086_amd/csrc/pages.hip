// Forks, plans, compaction and copies of pages that several sequences share (pages.h).
// All counts are integers, and what is decided by an order is decided by a maximum over row
// numbers, so that the results do not depend on which thread comes first.
#include <algorithm>

#include "pages.h"

namespace {

constexpr int NT = 256;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// pages of n tokens, and n as far as the table's row reaches
__device__ __forceinline__ int pages_of(int n, int psh) { return (int)(((long long)n + (1 << psh) - 1) >> psh); }

__device__ __forceinline__ bool in_pool(int p, int n_pages) { return (unsigned)p < (unsigned)n_pages; }

// entries of a that are refs as they were before the call
__device__ __forceinline__ void copy_ints(const int* from, int* to, long n, long gid, long gsz) {
  if (from == to) return;
  for (long i = gid; i < n; i += gsz) to[i] = from[i];
}

// ---------------------------------------------------------------------------
// Fork: row dst[i] lists the pages of the first len[i] tokens of row src[i], each with one
// holder more.  Every workgroup looks all forks over for itself (a bit per table row in
// LDS); the counts have to be in place before any is raised, hence a launch of their own
// where the caller keeps the old ones.
__global__ __launch_bounds__(NT) void pages_refs_kernel(const int* from, int* to, int n) {
  copy_ints(from, to, n, (long)blockIdx.x * NT + threadIdx.x, (long)gridDim.x * NT);
}

__global__ __launch_bounds__(NT) void pages_fork_kernel(PagesForkArgs a) {
  __shared__ unsigned rows[PAGES_MAX_TABLE / 32];
  __shared__ int bad;
  const int tid = threadIdx.x, lane = tid & 63;
  for (int i = tid; i < (a.n_rows + 31) / 32; i += NT) rows[i] = 0;
  if (tid == 0) bad = 0;
  __syncthreads();
  const long long cap = (long long)a.width << a.psh;
  for (int i = tid; i < a.n; i += NT) {
    const int s = a.src[i], d = a.dst[i], l = a.len[i];
    if ((unsigned)s >= (unsigned)a.n_rows || (unsigned)d >= (unsigned)a.n_rows || l < 0 || l > cap) bad = 1;
    else if (atomicOr(&rows[d >> 5], 1u << (d & 31)) >> (d & 31) & 1) bad = 1;      // two forks into one row
  }
  __syncthreads();
  if (!bad)
    for (int i = tid; i < a.n; i += NT)
      if (rows[a.src[i] >> 5] >> (a.src[i] & 31) & 1) bad = 1;                      // from a row that is forked into
  __syncthreads();
  const int b = bad;
  if (blockIdx.x == 0 && tid == 0) *a.status = b ? 2 : 0;
  if (b) return;
  for (int i = blockIdx.x * (NT / 64) + (tid >> 6); i < a.n; i += gridDim.x * (NT / 64)) {
    const int k = pages_of(a.len[i], a.psh);
    const int* s = a.table + (size_t)a.src[i] * a.width;
    int* d = a.table + (size_t)a.dst[i] * a.width;
    for (int j = lane; j < k; j += 64) {
      const int p = s[j];
      d[j] = p;
      if (in_pool(p, a.n_pages)) atomicAdd(&a.refs_out[p], 1);
    }
  }
}

// ---------------------------------------------------------------------------
// Plan.  With have = pages(len_old), want = pages(len_new) of a row:
//   drops    entries [want, have) of a row that shrinks: one holder less
//   a write  of a row that grows from inside its last page: where that page keeps other
//            holders, the row copies it, unless it is the last of the holders and all of them write
//   takes    a page for the copy, then want - have, from the ring's front
//   gives    dropped pages without a holder left, by the last row that dropped them, behind the ring's end
// Four launches (one of a small plan), each of which needs all of the one before: clear the notes (a page's drops
// and writers, the last row of them), note, decide per row, then place everything by prefix sums over
// the rows, which every workgroup of the last launch makes for itself.
constexpr int WRITER = PAGES_MAX_ROWS;      // a writer's row in `last`: above every row that drops

struct Lens {
  int o, n, have, want;
  bool ok;
};
__device__ __forceinline__ Lens lens_of(const PagesPlanArgs& a, int b) {
  Lens l;
  l.o = a.len_old[b];
  l.n = a.len_new[b];
  const long long cap = (long long)a.width << a.psh;
  l.ok = (l.o >= 0) & (l.n >= 0) & (l.o <= cap) & (l.n <= cap);
  l.have = l.ok ? pages_of(l.o, a.psh) : 0;
  l.want = l.ok ? pages_of(l.n, a.psh) : 0;
  return l;
}
// the row grows from inside a page
__device__ __forceinline__ bool writes_tail(const PagesPlanArgs& a, const Lens& l) {
  return l.ok && l.n > l.o && (l.o & ((1 << a.psh) - 1));
}

__global__ __launch_bounds__(NT) void pages_clear_kernel(PagesPlanArgs a) {
  const long gid = (long)blockIdx.x * NT + threadIdx.x, gsz = (long)gridDim.x * NT;
  for (long i = gid; i < a.n_pages; i += gsz) {
    a.todo[i] = 0;
    a.last[i] = -1;
  }
  if (gid == 0) *a.bad = 0;
  copy_ints(a.refs_in, a.refs_out, a.n_pages, gid, gsz);
  copy_ints(a.table_in, a.table_out, (long)a.batch * a.width, gid, gsz);
}

// by wave `w` of n
__device__ __forceinline__ void note(const PagesPlanArgs& a, int w, int n) {
  const int lane = threadIdx.x & 63;
  for (int b = w; b < a.batch; b += n) {
    const Lens l = lens_of(a, b);
    const int* row = a.table_in + (size_t)b * a.width;
    for (int j = l.want + lane; j < l.have; j += 64) {
      const int p = row[j];
      if (!in_pool(p, a.n_pages)) { *a.bad = 1; continue; }
      atomicAdd(&a.todo[p], 1);
      atomicMax(&a.last[p], b);
    }
    if (writes_tail(a, l) && lane == 0) {
      const int p = row[l.have - 1];
      if (!in_pool(p, a.n_pages)) { *a.bad = 1; continue; }
      atomicAdd(&a.todo[p], 1 << 16);
      atomicMax(&a.last[p], WRITER + b);
    }
  }
}

// holders of page p after the drops
__device__ __forceinline__ int holders(const PagesPlanArgs& a, int p) { return a.refs_in[p] - (a.todo[p] & 0xffff); }

// Whether row b, which drops page p, is the one that gives it back.  It leaves that as a note,
// which only this row looks at: the counts change in the next launch.
constexpr int GIVEN = -1;
__device__ __forceinline__ bool gives(const PagesPlanArgs& a, int b, int p) {
  if (!in_pool(p, a.n_pages) || a.last[p] != b || holders(a, p) > 0) return false;
  a.todo[p] = GIVEN;
  return true;
}

__device__ __forceinline__ void decide(const PagesPlanArgs& a, int w, int n) {
  const int lane = threadIdx.x & 63;
  for (int b = w; b < a.batch; b += n) {
    const Lens l = lens_of(a, b);
    const int* row = a.table_in + (size_t)b * a.width;
    int given = 0;
    for (int j0 = l.want; j0 < l.have; j0 += 64)
      given += __popcll(__ballot(j0 + lane < l.have && gives(a, b, row[j0 + lane])));
    int copies = 0;
    if (writes_tail(a, l)) {
      const int p = row[l.have - 1];
      if (in_pool(p, a.n_pages)) {
        const int r = holders(a, p), g = (unsigned)a.todo[p] >> 16;
        copies = r > 1 && !(g == r && a.last[p] == WRITER + b);
      }
    }
    if (lane == 0) {
      a.given[b] = given;
      a.copies[b] = copies;
    }
  }
}

__global__ __launch_bounds__(NT) void pages_note_kernel(PagesPlanArgs a) {
  note(a, blockIdx.x * (NT / 64) + (threadIdx.x >> 6), gridDim.x * (NT / 64));
}
__global__ __launch_bounds__(NT) void pages_decide_kernel(PagesPlanArgs a) {
  decide(a, blockIdx.x * (NT / 64) + (threadIdx.x >> 6), gridDim.x * (NT / 64));
}
__device__ __forceinline__ long long scan64(long long v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long t = __shfl_up(v, o, 64);
    if (lane >= o) v += t;
  }
  return v;
}

// largest b in [0, n) with off[b] <= v
__device__ __forceinline__ int find_row(const int* off, int n, int v) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (off[mid] <= v) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// sh: 3 (B + 1) ints of LDS; by workgroup `me` of n, of N threads
template <int N> __device__ __forceinline__ void place(const PagesPlanArgs& a, int* sh, int me, int n) {
  const int B = a.batch, tid = threadIdx.x, lane = tid & 63, T = 1 << a.psh;
  int *taken = sh, *given = sh + (B + 1), *rows = sh + 2 * (B + 1);    // exclusive sums
  __shared__ long long part[3][N / 64];
  __shared__ int bad_len;
  if (tid == 0) bad_len = 0;
  __syncthreads();
  const int per = (B + N - 1) / N, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  long long st = 0, sg = 0, sr = 0;
  for (int b = b0; b < b1; ++b) {
    const Lens l = lens_of(a, b);
    if (!l.ok) bad_len = 1;
    st += a.copies[b] + max(l.want - l.have, 0);
    sg += a.given[b];
    sr += l.ok ? max((long long)l.n - l.o, 0LL) : 0;
  }
  const int w = tid >> 6;
  const long long it = scan64(st), ig = scan64(sg), ir = scan64(sr);
  if (lane == 63) { part[0][w] = it; part[1][w] = ig; part[2][w] = ir; }
  __syncthreads();
  long long bt = it - st, bg = ig - sg, br = ir - sr, tt = 0, tg = 0, tr = 0;
#pragma unroll
  for (int i = 0; i < N / 64; ++i) {
    if (i < w) { bt += part[0][i]; bg += part[1][i]; br += part[2][i]; }
    tt += part[0][i]; tg += part[1][i]; tr += part[2][i];
  }
  const int head = a.pool_in[0], count = a.pool_in[1];
  int status = 0;
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) status = 4;
  else if (bad_len) status = 2;
  else if (*a.bad || tg > a.n_pages - count) status = 4;
  else if (tt > count) status = 1;
  else if (tr > a.slot_rows) status = 3;
  const int total = status ? 0 : (int)tr;
  if (!status) {
    for (int b = b0; b < b1; ++b) {
      const Lens l = lens_of(a, b);
      taken[b] = (int)bt;
      given[b] = (int)bg;
      rows[b] = (int)br;
      bt += a.copies[b] + max(l.want - l.have, 0);
      bg += a.given[b];
      br += max(l.n - l.o, 0);
    }
    if (tid == 0) { taken[B] = (int)tt; given[B] = (int)tg; rows[B] = (int)tr; }
  }
  __syncthreads();

  auto ring = [&](int i) __attribute__((always_inline)) {
    const unsigned k = (unsigned)head + (unsigned)i, n = (unsigned)a.n_pages;
    return k >= n ? k - n : k;
  };
  const int gid = me * N + tid, gsz = n * N;
  if (gid == 0) {
    *a.status = status;
    a.pool_out[0] = status ? head : (int)ring((int)tt);
    a.pool_out[1] = status ? count : (int)(count - tt + tg);
  }
  for (int b = gid; b <= B; b += gsz) a.row_off[b] = status ? 0 : rows[b];
  // copies, with the entry that changes
  for (int b = gid; b < B; b += gsz) {
    int from = -1, to = -1;
    if (!status && a.copies[b]) {
      const size_t at = (size_t)b * a.width + pages_of(a.len_old[b], a.psh) - 1;
      from = a.table_in[at];
      to = a.free_pages[ring(taken[b])];
      a.table_out[at] = to;
      atomicSub(&a.refs_out[from], 1);
      if (in_pool(to, a.n_pages)) a.refs_out[to] = 1;
    }
    a.copy_src[b] = from;
    a.copy_dst[b] = to;
  }
  if (!status) {
    // pages taken, the copies' left out
    for (int r = gsz - 1 - gid; r < (int)tt; r += gsz) {
      const int b = find_row(taken, B, r), i = r - taken[b] - a.copies[b];
      if (i < 0) continue;
      const int p = a.free_pages[ring(r)];
      a.table_out[(size_t)b * a.width + pages_of(a.len_old[b], a.psh) + i] = p;
      if (in_pool(p, a.n_pages)) a.refs_out[p] = 1;
    }
    // drops: a wave a row
    for (int b = gsz / 64 - 1 - gid / 64; b < B; b += gsz / 64) {
      const Lens l = lens_of(a, b);
      const int* row = a.table_in + (size_t)b * a.width;
      int at = given[b];
      for (int j0 = l.want; j0 < l.have; j0 += 64) {
        const bool in = j0 + lane < l.have;
        const int p = row[min(j0 + lane, l.have - 1)];
        const bool mine = in && a.last[p] == b && a.todo[p] == GIVEN;
        const unsigned long long m = __ballot(mine);
        if (mine) a.free_pages[ring(count + at + __popcll(m & ((1ull << lane) - 1)))] = p;
        at += __popcll(m);
        if (in) atomicSub(&a.refs_out[p], 1);
      }
    }
  }
  for (long long r = gid; r < a.slot_rows; r += gsz) {
    int s = -1;
    if (r < total) {
      const int b = find_row(rows, B, (int)r), o = a.len_old[b], have = pages_of(o, a.psh);
      const int p = o + (int)r - rows[b], j = p >> a.psh, c = a.copies[b];
      if (j < have - c) s = a.table_in[(size_t)b * a.width + j];
      else s = a.free_pages[ring(taken[b] + j - have + c)];
      s = in_pool(s, a.n_pages) ? (s << a.psh) + (p & (T - 1)) : -1;
    }
    a.slots[r] = s;
  }
}
__global__ __launch_bounds__(NT) void pages_place_kernel(PagesPlanArgs a) {
  extern __shared__ int sh[];
  place<NT>(a, sh, blockIdx.x, gridDim.x);
}
// A small plan by one workgroup, a row to a wave, its notes in LDS (16 rows of 4096 pages: 8.9 us, in four
// launches 11.5; 8 rows that take 16384 slots 9.4 and 10.4).
constexpr int PLAN_NT = 1024, PLAN_PAGES = 4096, PLAN_BATCH = PLAN_NT / 64, PLAN_SLOTS = 16384;
__global__ __launch_bounds__(PLAN_NT) void pages_small_kernel(PagesPlanArgs a) {
  __shared__ int todo[PLAN_PAGES], last[PLAN_PAGES], sums[3 * (PLAN_BATCH + 1)], bad;
  const int tid = threadIdx.x;
  a.todo = todo;
  a.last = last;
  a.bad = &bad;
  for (int i = tid; i < a.n_pages; i += PLAN_NT) {
    todo[i] = 0;
    last[i] = -1;
  }
  if (tid == 0) bad = 0;
  copy_ints(a.refs_in, a.refs_out, a.n_pages, tid, PLAN_NT);
  copy_ints(a.table_in, a.table_out, (long)a.batch * a.width, tid, PLAN_NT);
  __syncthreads();
  note(a, tid >> 6, PLAN_NT / 64);
  __syncthreads();
  decide(a, tid >> 6, PLAN_NT / 64);
  __syncthreads();
  place<PLAN_NT>(a, sums, 0, 1);
}

// ---------------------------------------------------------------------------
// Compaction.  U pages are in use.  Those from U on, in rising order, move to the free ones
// below U, in rising order: there are as many of both.  The moves of a page are found by
// prefix sums over the pages: a launch counts the pages in use of each block, and each
// workgroup of the next one adds the blocks up for itself (of up to COUNTED pages it counts them itself: 8192 pages 12.6 us,
// 8193 in three launches 13.5); a third one rewrites the tables.
constexpr int COUNTED = 4 * PAGES_BLOCK;
__device__ __forceinline__ int block_sum_int(int v, int* red) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) t += red[i];
  return t;
}

__global__ __launch_bounds__(NT) void pages_used_kernel(PagesCompactArgs a) {
  __shared__ int red[NT / 64];
  const long p0 = (long)blockIdx.x * PAGES_BLOCK;
  int n = 0;
#pragma unroll
  for (int i = 0; i < PAGES_BLOCK / NT; ++i) {
    const long p = p0 + i * NT + threadIdx.x;
    n += p < a.n_pages && a.refs_in[p] > 0;
  }
  n = block_sum_int(n, red);
  if (threadIdx.x == 0) a.used[blockIdx.x] = n;
}

__global__ __launch_bounds__(NT) void pages_moves_kernel(PagesCompactArgs a) {
  __shared__ int red[NT / 64], wsum[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, nb = gridDim.x, me = blockIdx.x;
  // pages in use in all, before this block, and below U: blocks before U's, then its part of that block
  int all = 0, mine = 0, below = 0;
  if (a.n_pages <= COUNTED) {
#pragma unroll 8
    for (int p = tid; p < a.n_pages; p += NT) {
      const int n = a.refs_in[p] > 0;
      all += n;
      mine += p < me * PAGES_BLOCK ? n : 0;
    }
  } else {
    for (int i = tid; i < nb; i += NT) {
      const int n = a.used[i];
      all += n;
      mine += i < me ? n : 0;
    }
  }
  const int U = block_sum_int(all, red);
  mine = block_sum_int(mine, red);
  const int ub = a.n_pages <= COUNTED ? 0 : U / PAGES_BLOCK;
  for (int i = tid; i < min(ub, nb); i += NT) below += a.used[i];
#pragma unroll 8
  for (int p = ub * PAGES_BLOCK + tid; p < U; p += NT) below += a.refs_in[p] > 0;
  below = block_sum_int(below, red);
  const int moves = U - below;
  if (me == 0 && tid == 0) {
    *a.moves = moves;
    a.pool_out[0] = 0;
    a.pool_out[1] = a.n_pages - U;
  }
  // 8 consecutive pages a thread
  constexpr int E = PAGES_BLOCK / NT;
  const long p0 = (long)me * PAGES_BLOCK + tid * E;
  int ref[E], n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    ref[e] = p0 + e < a.n_pages ? a.refs_in[p0 + e] : 0;
    n += ref[e] > 0;
  }
  const int incl = (int)scan64(n);
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int before = mine + incl - n;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i)
    if (i < w) before += wsum[i];
  const int half = a.n_pages / 2;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long p = p0 + e;
    if (p >= a.n_pages) break;
    const bool u = ref[e] > 0;
    int rank = -1;
    if (u && p >= U) a.move_src[rank = before - below] = (int)p;
    if (!u && p < U) a.move_dst[(int)p - before] = (int)p;
    a.rank[p] = rank;
    a.free_pages[p] = p < a.n_pages - U ? U + (int)p : -1;
    if (a.refs_out != a.refs_in) a.refs_out[p] = ref[e];
    if (p >= moves && p < half) a.move_src[p] = a.move_dst[p] = -1;
    before += u;
  }
}

__global__ __launch_bounds__(NT) void pages_remap_kernel(PagesCompactArgs a) {
  const long gid = (long)blockIdx.x * NT + threadIdx.x, gsz = (long)gridDim.x * NT;
  const int moves = *a.moves;
  for (long r = gid; r < moves; r += gsz) {
    const int s = a.move_src[r], d = a.move_dst[r];
    a.refs_out[d] = a.refs_in[s];
    a.refs_out[s] = 0;
  }
  for (long i = gid; i < (long)a.batch * a.width; i += gsz) {
    const int b = (int)(i / a.width), j = (int)(i % a.width);
    const int n = min(max(a.len[b], 0), (int)min((long long)a.width << a.psh, 0x7fffffffLL));
    int p = a.table_in[i];
    const bool held = j < pages_of(n, a.psh) && in_pool(p, a.n_pages);
    if (held && a.rank[p] >= 0) p = a.move_dst[a.rank[p]];
    else if (a.table_out == a.table_in) continue;
    a.table_out[i] = p;
  }
}

// ---------------------------------------------------------------------------
// Copy of whole pages, in 16-byte pieces: a workgroup takes COPY bytes of a page at a time.
// Entries outside the pool are passed over.  Bound by the memory, bytes read and written.
constexpr int COPY = 16 * 4 * NT;

__global__ __launch_bounds__(NT) void pages_copy_kernel(PagesCopyArgs a) {
  const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  const long chunks = (a.page_bytes + COPY - 1) / COPY, items = chunks * n * a.planes;
  for (long i = blockIdx.x; i < items; i += gridDim.x) {
    const long e = i / chunks, c = i % chunks;
    const int k = (int)(e % n), s = a.src[k], d = a.dst[k];
    if (!in_pool(s, a.n_pages) || !in_pool(d, a.n_pages)) continue;
    char* plane = a.data + (e / n) * a.plane_stride;
    const u32x4* from = (const u32x4*)(plane + s * a.page_bytes);
    u32x4* to = (u32x4*)(plane + d * a.page_bytes);
    const long q0 = c * (COPY / 16) + threadIdx.x, q1 = a.page_bytes / 16;
    u32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = from[min(q0 + u * NT, q1 - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (q0 + u * NT < q1) to[q0 + u * NT] = x[u];
  }
}

unsigned blocks(long items, long most) { return (unsigned)std::min(std::max((items + NT - 1) / NT, 1L), most); }

}  // namespace

void launch_pages_fork(const PagesForkArgs& a, hipStream_t st) {
  if (a.refs_in != a.refs_out) pages_refs_kernel<<<blocks(a.n_pages, 1024), NT, 0, st>>>(a.refs_in, a.refs_out, a.n_pages);
  pages_fork_kernel<<<blocks((long)a.n * 64, 256), NT, 0, st>>>(a);
}

void launch_pages_plan(const PagesPlanArgs& a, hipStream_t st) {
  const long table = a.table_in == a.table_out ? 0 : (long)a.batch * a.width;
  if (a.n_pages <= PLAN_PAGES && a.batch <= PLAN_BATCH && table <= 4 * PLAN_PAGES && a.slot_rows <= PLAN_SLOTS) {
    pages_small_kernel<<<1, PLAN_NT, 0, st>>>(a);
    return;
  }
  pages_clear_kernel<<<blocks(std::max((long)a.n_pages, table), 1024), NT, 0, st>>>(a);
  pages_note_kernel<<<blocks((long)a.batch * 64, 1024), NT, 0, st>>>(a);
  pages_decide_kernel<<<blocks((long)a.batch * 64, 1024), NT, 0, st>>>(a);
  const long items = std::max((long)a.slot_rows, (long)a.batch * 64);
  pages_place_kernel<<<blocks(items, 512), NT, 3 * (a.batch + 1) * sizeof(int), st>>>(a);
}

void launch_pages_compact(const PagesCompactArgs& a, hipStream_t st) {
  const unsigned nb = (unsigned)(((long)a.n_pages + PAGES_BLOCK - 1) / PAGES_BLOCK);
  if (a.n_pages > COUNTED) pages_used_kernel<<<nb, NT, 0, st>>>(a);
  pages_moves_kernel<<<nb, NT, 0, st>>>(a);
  pages_remap_kernel<<<blocks(std::max((long)a.batch * a.width, (long)a.n_pages / 2), 1024), NT, 0, st>>>(a);
}

void launch_pages_copy(const PagesCopyArgs& a, hipStream_t st) {
  const long items = (a.page_bytes + COPY - 1) / COPY * a.n * a.planes;
  pages_copy_kernel<<<(unsigned)std::min(items, 4096L), NT, 0, st>>>(a);
}
