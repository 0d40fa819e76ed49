// Sampling of a token per row of logits, from given random numbers:
//   z = l / T,  w = exp(z - max z),  tokens ordered by falling logit, then by rising index
//   S1 = the first top_k tokens, S2 = the shortest prefix of S1 with at least top_p of S1's weight,
//   S3 = the tokens with w >= min_p; kept are S2 and S3 together, the first token always
//   token = the first one, in the vocabulary's order, at which the kept weight summed so far exceeds u times all of it
//
// A drawn token changes where a sum crosses a border, so weights are computed and summed in 64 bits, by fixed
// orders or in integers: the same bits whatever order the waves run in.
//
// A workgroup has a row.  With t = 16 (l - m0) / T, m0 a reference near the row's maximum, the weight
// relative to m0 is
//   w = E[b] e^x,  b = floor(t),  x = (t - b - 1/2) / 16 in [-1/32, 1/32),  E[b] = exp((b + 1/2) / 16)
// e^x by 8 terms of its series (2^-55), E from a table in LDS.  The bins b are at the same time those of a
// histogram, of e^x in units of 2^-44 (and of tokens, where top_k asks for them): its one pass over the row
// gives the bin at which each filter cuts.  Another pass collects the tokens of the bins from there on
// into LDS, where they are sorted and drawn from.  Where these are too many the tokens of the bin of the cut alone are
// collected, for the cut itself, and the sums of the kept weights of each wave's share of the row made, to
// draw from by descending to a sixteenth of it.
//   Tokens 33 and more nats below m0 have no bin (2^-47 of the largest weight); where one is 95 above, m0 was
//   too low, and the pass is made again with the row's maximum.
#include <algorithm>

#include "sample.h"

namespace {

constexpr int BINS = 2048, BELOW = 33 * 16;      // bins, and those below m0
constexpr int LIST = 2048;                       // tokens that are sorted in LDS
constexpr double UNIT = 17592186044416.0;        // 2^44

// bits whose order as unsigned is that of the floats; -0 like 0
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <class T> struct Vec { static constexpr int N = 16 / sizeof(T); };

template <int NT> struct Shared {
  unsigned long long mass[BINS];
  double edge[BINS];
  unsigned count[BINS];
  unsigned long long list[LIST];
  double weight[LIST];
  double seg[NT / 64];
  double redd[NT / 64];
  long long redi[NT / 64];
  double cut;
  unsigned long long found;
  int n, flag;
};

// w relative to m0 is edge[bin] * e^x
struct Place {
  int bin;       // outside [0, BINS): below or above every bin
  double ex;
};
__device__ __forceinline__ Place place_of(float l, double m0, double inv16) {
  const double t = ((double)l - m0) * inv16, f = floor(t);
  Place p;
  const double x = fma(t - f, 1.0 / 16, -1.0 / 32);
  double e = 1.0 / 5040;
  e = fma(e, x, 1.0 / 720);
  e = fma(e, x, 1.0 / 120);
  e = fma(e, x, 1.0 / 24);
  e = fma(e, x, 1.0 / 6);
  e = fma(e, x, 0.5);
  e = fma(e, x, 1.0);
  p.ex = fma(e, x, 1.0);
  p.bin = (int)fmin(fmax(f, -1e6), 1e6) + BELOW;
  return p;
}

template <class T, int NT> struct Row {
  static constexpr int NW = NT / 64, N = Vec<T>::N;
  const SampleArgs& a;
  Shared<NT>& s;
  const T* row;
  const int tid, lane, w;
  int V, share;              // a wave's share of the row: tokens w share .. + share - 1
  bool inf;                  // the row's maximum is infinite: its tokens alone, alike
  double m0, inv16;

  __device__ Row(const SampleArgs& a, Shared<NT>& s, int r)
      : a(a), s(s), row((const T*)a.logits + (size_t)r * a.ld), tid(threadIdx.x), lane(tid & 63),
        w(__builtin_amdgcn_readfirstlane(tid >> 6)), V(a.vocab), inf(false) {
    share = (V + NW - 1) / NW;
    share = (share + 64 * N - 1) / (64 * N) * (64 * N);
  }

  __device__ __forceinline__ float logit(float x, int i) const {
    if (i == a.exclude) return -INFINITY;
    return inf ? (x == INFINITY ? 0.f : x != x ? x : -INFINITY) : x;
  }

  // f(logit, index) for the tokens [i0, i1), by the calling wave: 16 bytes a lane, U loads at a time
  template <class F> __device__ __forceinline__ void tokens(int i0, int i1, F&& f) const {
    constexpr int U = 4;
    i1 = min(i1, V);
    if (V < N) {
      for (int i = i0 + lane; i < i1; i += 64) f(logit(to_f32(row[i]), i), i);
      return;
    }
    for (int i = i0; i < i1; i += 64 * N * U) {
      T x[U][N];
      int at[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        at[u] = i + (u * 64 + lane) * N;
        __builtin_memcpy(x[u], row + min(at[u], V - N), 16);     // past the end: the last ones
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int back = max(at[u] - (V - N), 0);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int k = at[u] - back + e;
          if (k >= at[u] && k < i1) f(logit(to_f32(x[u][e]), k), k);
        }
      }
    }
  }
  template <class F> __device__ __forceinline__ void all_tokens(F&& f) const { tokens(w * share, (w + 1) * share, f); }

  // ---- reductions over the workgroup; every thread gets the result
  __device__ double sum(double x) {
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) s.redd[w] = x;
    __syncthreads();
    double t = 0;
    for (int i = 0; i < NW; ++i) t += s.redd[i];
    return t;
  }
  __device__ long long max_all(long long x) {
    for (int o = 32; o; o >>= 1) x = max(x, (long long)__shfl_xor(x, o, 64));
    __syncthreads();
    if (lane == 0) s.redi[w] = x;
    __syncthreads();
    long long t = s.redi[0];
    for (int i = 1; i < NW; ++i) t = max(t, s.redi[i]);
    return t;
  }
  __device__ bool any(bool x) { return max_all(x) != 0; }
  // inclusive sums over the threads, in thread order
  template <class X> __device__ X scan(X x, X* red) {
    for (int o = 1; o < 64; o <<= 1) {
      const X y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) red[w] = x;
    __syncthreads();
    X before = 0;
    for (int i = 0; i < w; ++i) before += red[i];
    return x + before;
  }

  __device__ __forceinline__ Place place(float l) const { return place_of(l, m0, inv16); }
  __device__ __forceinline__ double weight(float l) const {
    const Place p = place(l);
    return p.bin >= 0 && l > -INFINITY ? s.edge[min(p.bin, BINS - 1)] * p.ex : 0.0;
  }
  __device__ __forceinline__ int bin(float l) const { return l > -INFINITY ? place(l).bin : -1; }

  // ---- what is kept: tokens whose (key, index) comes no later than the cut
  struct Cut {
    unsigned key;       // tokens of greater keys are kept, of this one those up to index `last`
    int last;
    __device__ __forceinline__ bool keeps(float l, int i) const {
      const unsigned k = key_of(l);
      return k > key || (k == key && i <= last);
    }
  };

  // Sums of the kept weights of each wave's share, in s.seg; returns all of it.
  __device__ double shares(const Cut& c) {
    double x = 0;
    all_tokens([&](float l, int i) { x += c.keeps(l, i) ? weight(l) : 0.0; });
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) s.seg[w] = x;
    __syncthreads();
    double t = 0;
    for (int i = 0; i < NW; ++i) t += s.seg[i];
    return t;
  }

  // The token at which the kept weight exceeds u times all of it, from the shares' sums: descend into the share,
  // then into a wave's part of it, then token by token.
  __device__ void draw_from_shares(const Cut& c, double total, double u, int r) {
    double target = u * total, before = 0;
    int at = -1, some = 0;
    for (int i = 0; i < NW; ++i) {
      if (s.seg[i] > 0) some = i;
      if (at < 0 && before + s.seg[i] > target) at = i;
      if (at < 0) before += s.seg[i];
    }
    if (at < 0) {               // u near one and the sums' rounding: the last weight there is
      at = some;
      before = total - s.seg[some];
      target = total * 2;
    }
    const int i0 = at * share, part = (share / NW + 64 * N - 1) / (64 * N) * (64 * N);
    double x = 0;
    tokens(i0 + w * part, min(i0 + (w + 1) * part, i0 + share), [&](float l, int i) { x += c.keeps(l, i) ? weight(l) : 0.0; });
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) s.redd[w] = x;
    __syncthreads();
    int in = -1;
    some = 0;
    for (int i = 0; i < NW; ++i) {
      if (s.redd[i] > 0) some = i;
      if (in < 0 && before + s.redd[i] > target) in = i;
      if (in < 0) before += s.redd[i];
    }
    if (in < 0) {
      in = some;
      before -= s.redd[some];
    }
    if (w != 0) return;
    // one wave: 64 tokens at a time, in order
    int token = -1;
    double wt = 0;
    const int p0 = i0 + in * part, p1 = min(min(p0 + part, i0 + share), V);
    for (int p = p0; p < p1; p += 64) {
      const int i = p + lane;
      const float l = i < p1 ? logit(to_f32(row[i]), i) : -INFINITY;
      const double x = i < p1 && c.keeps(l, i) ? weight(l) : 0.0;
      double y = x;
      for (int o = 1; o < 64; o <<= 1) {
        const double z = __shfl_up(y, o, 64);
        if (lane >= o) y += z;
      }
      const unsigned long long hit = __ballot(x > 0 && before + y > target), pos = __ballot(x > 0);
      const unsigned long long m = hit ? hit : pos;
      if (m) {
        const int k = hit ? __ffsll((unsigned long long)hit) - 1 : 63 - __clzll((long long)pos);
        token = p + k;
        wt = __shfl(x, k, 64);
      }
      if (hit) break;
      before += __shfl(y, 63, 64);
    }
    if (lane == 0) write(r, token, (float)log(wt / total));
  }

  __device__ void write(int r, int token, float logp) {
    a.token[r] = token;
    if (a.logp) a.logp[r] = logp;
  }

  // ---- the first pass
  // Histogram of the row (or, without filters, the shares' sums) about m0; the row's maximum key, with
  // its first index, in `best`.  False: m0 has to be raised to the maximum.
  __device__ bool survey(bool hist, bool counts, unsigned long long& best, bool& nan) {
    for (int i = tid; i < BINS; i += NT) {
      s.mass[i] = 0;
      s.count[i] = 0;
      s.edge[i] = exp((i - BELOW + 0.5) / 16);
    }
    __syncthreads();
    unsigned long long top = 0;
    double x = 0;
    bool bad = false, high = false;
    all_tokens([&](float l, int i) {
      bad |= l != l;
      const unsigned long long k = (unsigned long long)key_of(l) << 32 | (unsigned)~i;
      top = k > top ? k : top;
      const Place p = place(l);
      high |= p.bin >= BINS;
      if (p.bin >= 0 && p.bin < BINS && l > -INFINITY) {
        if (hist) {
          atomicAdd(&s.mass[p.bin], (unsigned long long)(p.ex * UNIT));
          if (counts) atomicAdd(&s.count[p.bin], 1u);
        } else {
          x += s.edge[p.bin] * p.ex;
        }
      }
    });
    best = (unsigned long long)max_all((long long)(top ^ 1ull << 63)) ^ 1ull << 63;
    nan = any(bad);
    if (!hist) {
      for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
      if (lane == 0) s.seg[w] = x;
    }
    const bool again = any(high);
    return !again;
  }

  // ---- the tokens for which pick holds, into the list; their number, which may be more than fit
  template <class P> __device__ int collect(P&& pick) {
    if (tid == 0) s.n = 0;
    __syncthreads();
    all_tokens([&](float l, int i) {
      if (pick(l, i)) {
        const int at = atomicAdd(&s.n, 1);
        if (at < LIST) s.list[at] = (unsigned long long)~key_of(l) << 32 | (unsigned)i;
      }
    });
    __syncthreads();
    return s.n;
  }

  // s.list[0 .. n) in rising order
  __device__ void sort(int n) {
    int m = 2;
    while (m < n) m *= 2;
    for (int i = n + tid; i < m; i += NT) s.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= m; k *= 2)
      for (int j = k / 2; j; j /= 2) {
        for (int i = tid; i < m / 2; i += NT) {
          const int lo = (i / j) * 2 * j + i % j, hi = lo + j;
          const unsigned long long x = s.list[lo], y = s.list[hi];
          if ((x > y) == ((lo & k) == 0)) {
            s.list[lo] = y;
            s.list[hi] = x;
          }
        }
        __syncthreads();
      }
  }
  __device__ __forceinline__ float list_logit(int i) const { return value_of(~(unsigned)(s.list[i] >> 32)); }

  // Inclusive sums of the list's weights, in its order, in s.weight.
  __device__ void list_sums(int n) {
    constexpr int E = LIST / NT;
    double x[E], t = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = tid * E + e;
      x[e] = i < n ? weight(list_logit(i)) : 0.0;
      t += x[e];
    }
    double y = scan(t, s.redd) - t;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      y += x[e];
      s.weight[tid * E + e] = y;
    }
    __syncthreads();
  }

  // number of i < n with f(i), which falls from true to false: by all threads
  template <class F> __device__ int count_list(int n, F&& f) {
    int c = 0;
    for (int i = tid; i < n; i += NT) c += f(i);
    return (int)sum((double)c);
  }

  // The list holds the first n tokens of the order: filters and draw in LDS.
  __device__ void finish_list(int n, int k, double p, double floor_l, double mass1, double u, int r) {
    sort(n);
    list_sums(n);
    int kept = n;
    if (k > 0) kept = min(kept, k);
    if (p < 1) {
      const double all = k > 0 ? s.weight[min(k, n) - 1] : mass1, most = p * all;
      kept = min(kept, max(1, count_list(n, [&](int i) { return (i ? s.weight[i - 1] : 0.0) < most; })));
    }
    if (floor_l > -INFINITY) kept = min(kept, max(1, count_list(n, [&](int i) { return (double)list_logit(i) >= floor_l; })));
    // once more in the vocabulary's order
    __syncthreads();
    for (int i = tid; i < kept; i += NT) s.list[i] = (s.list[i] << 32) | (~(unsigned)(s.list[i] >> 32));
    __syncthreads();
    sort(kept);
    for (int i = tid; i < kept; i += NT) s.list[i] = (unsigned long long)~(unsigned)s.list[i] << 32 | (unsigned)(s.list[i] >> 32);
    __syncthreads();
    list_sums(kept);
    const double total = s.weight[kept - 1], target = u * total;
    const int at = min(count_list(kept, [&](int i) { return s.weight[i] <= target; }), kept - 1);
    // (a token of weight zero is never the first above a border; the last of the list may be one)
    if (tid == 0) {
      int i = at;
      while (i > 0 && weight(list_logit(i)) == 0) --i;
      write(r, (int)(unsigned)s.list[i], (float)log(weight(list_logit(i)) / total));
    }
  }

  // ---- cuts of many tokens
  // The bin, from the highest on, in which the sum of f over the bins reaches `target`, and the sum above it;
  // -1 where it is not reached.
  template <class F> __device__ int cross(double target, double& above, F&& f) {
    constexpr int E = BINS / NT;
    double x[E], t = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = f(BINS - 1 - (tid * E + e));
      t += x[e];
    }
    double y = scan(t, s.redd) - t;
    if (tid == 0) s.flag = -1;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (y < target && y + x[e] >= target) {
        s.flag = BINS - 1 - (tid * E + e);
        s.cut = y;
      }
      y += x[e];
    }
    __syncthreads();
    const int b = s.flag;
    above = s.cut;
    __syncthreads();
    return b;
  }

  // Smallest key of a logit whose bin is at least b.
  __device__ unsigned first_key(int b) const {
    unsigned lo = key_of(-INFINITY) + 1, hi = key_of(INFINITY);      // bin(hi) >= b
    while (lo < hi) {
      const unsigned mid = lo + (hi - lo) / 2;
      if (bin(value_of(mid)) >= b) hi = mid; else lo = mid + 1;
    }
    return lo;
  }

  // The cut within bin b: the tokens of higher bins amount to `above`, the cut is where `target` is reached.
  // by_count: tokens are counted, else their weights summed.
  __device__ Cut cut_in_bin(int b, double above, double target, bool by_count) {
    unsigned lo = first_key(b), hi = b + 1 < BINS ? first_key(b + 1) - 1 : key_of(INFINITY);
    for (;;) {
      const unsigned klo = lo, khi = hi;
      const int n = collect([&](float l, int) { const unsigned k = key_of(l); return k >= klo && k <= khi && l > -INFINITY; });
      if (n <= LIST) {
        sort(n);
        list_sums(n);
        const int kept = min(n, max(1, count_list(n, [&](int i) {
          return above + (by_count ? (double)i : i ? s.weight[i - 1] : 0.0) < target; })));
        const unsigned long long e = s.list[kept - 1];
        __syncthreads();
        return Cut{~(unsigned)(e >> 32), (int)(unsigned)e};
      }
      if (lo == hi) {                    // one value, more often than the list holds: its first tokens
        const double each = by_count ? 1.0 : weight(value_of(lo));
        const long long want = min((long long)max(1.0, ceil((target - above) / each)), (long long)n);
        return Cut{lo, nth(lo, (int)want)};
      }
      // 2048 parts of the keys
      int shift = 0;
      while ((hi - lo) >> shift >= BINS) ++shift;
      for (int i = tid; i < BINS; i += NT) s.mass[i] = s.count[i] = 0;
      __syncthreads();
      all_tokens([&](float l, int) {
        const unsigned k = key_of(l);
        if (k < klo || k > khi || !(l > -INFINITY)) return;
        const int i = (k - klo) >> shift;
        atomicAdd(&s.count[i], 1u);
        if (!by_count) atomicAdd(&s.mass[i], (unsigned long long)(place(l).ex * UNIT));
      });
      __syncthreads();
      const double e = s.edge[b] / UNIT;
      const double rest = target - above;
      double more = 0;
      int i = cross(rest, more, [&](int k) { return by_count ? (double)s.count[k] : (double)s.mass[k] * e; });
      if (i < 0) {                       // not reached, by rounding: the lowest part that has a token
        i = cross(1e-300, more, [&](int k) { return s.count[BINS - 1 - k] ? 1.0 : 0.0; });
        i = BINS - 1 - max(i, 0);
        more = rest;
      }
      above += more;
      lo += (unsigned)i << shift;
      hi = min(hi, lo + (1u << shift) - 1);
    }
  }

  // Index of the n-th token of this key.
  __device__ int nth(unsigned key, int n) {
    int c = 0;
    all_tokens([&](float l, int) { c += key_of(l) == key; });
    for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o, 64);
    __syncthreads();
    if (lane == 0) s.redi[w] = c;
    __syncthreads();
    int at = 0;
    while (at < NW - 1 && n > (int)s.redi[at]) n -= (int)s.redi[at++];
    __syncthreads();
    if (w == 0) {
      const int p1 = min((at + 1) * share, V);
      int res = p1 - 1;
      for (int p = at * share; p < p1; p += 64) {
        const int i = p + lane;
        const unsigned long long m = __ballot(i < p1 && key_of(logit(to_f32(row[min(i, V - 1)]), i)) == key);
        const int k = __popcll(m);
        if (n <= k) {
          const unsigned long long me = __ballot((m >> lane & 1) && __popcll(m & ((2ull << lane) - 1)) == n);
          res = p + __ffsll(me) - 1;
          break;
        }
        n -= k;
      }
      if (lane == 0) s.flag = res;
    }
    __syncthreads();
    const int i = s.flag;
    __syncthreads();
    return i;
  }
};

template <class T, int NT>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
  __shared__ Shared<NT> s;
  const int r = blockIdx.x, tid = threadIdx.x;
  Row<T, NT> row(a, s, r);
  const float temp = a.temperature ? a.temperature[r] : 1.f;
  const int want_k = a.top_k ? a.top_k[r] : 0;
  const double p = a.top_p ? (double)a.top_p[r] : 1.0, mp = a.min_p ? (double)a.min_p[r] : 0.0;
  const float uf = a.u[r];
  const double u = uf > 0.f ? (double)uf : 0.0;
  const bool greedy = !(temp > 0.f);
  const int k = want_k > 0 && want_k < a.vocab ? want_k : 0;
  const bool by_p = p < 1, by_m = mp > 0, filters = k || by_p || by_m;

  // the reference: the maximum of a few tokens, 0 where these are none
  unsigned long long best = 0;
  {
    unsigned top = 0;
    row.tokens(row.w * 64 * Vec<T>::N, (row.w + 1) * 64 * Vec<T>::N, [&](float l, int) {
      if (l < INFINITY) top = max(top, key_of(l));
    });
    const unsigned t = (unsigned)row.max_all(top);
    row.m0 = t > key_of(-INFINITY) ? (double)value_of(t) : 0.0;
  }
  row.inv16 = greedy ? 0.0 : 16.0 / (double)temp;
  bool nan = false;
  for (;;) {
    const bool fits = row.survey(filters && !greedy, k != 0, best, nan);
    if (nan) {
      if (tid == 0) row.write(r, -1, NAN);
      return;
    }
    const float top = value_of((unsigned)(best >> 32));
    if (top == -INFINITY) {              // no token at all
      if (tid == 0) row.write(r, -1, -INFINITY);
      return;
    }
    if (greedy) {
      if (tid == 0) row.write(r, (int)~(unsigned)best, 0.f);
      return;
    }
    if (top == INFINITY) {               // infinite logits share the whole weight
      row.inf = true;
      row.m0 = 0;
      continue;
    }
    if (fits && row.m0 <= (double)top) break;      // (above it: the few tokens were none)
    row.m0 = (double)top;
  }
  const double top = (double)value_of((unsigned)(best >> 32));
  using Cut = typename Row<T, NT>::Cut;
  Cut cut{key_of(-INFINITY), -1};        // everything
  if (!filters) {
    __syncthreads();
    double total = 0;
    for (int i = 0; i < NT / 64; ++i) total += s.seg[i];
    row.draw_from_shares(cut, total, u, r);
    return;
  }
  if (p <= 0 || mp > 1) {                // the first token alone
    if (tid == 0) row.write(r, (int)~(unsigned)best, 0.f);
    return;
  }
  // a token is kept by min_p where its logit is no lower than this
  const double floor_l = by_m ? top + (mp < 1 ? log(mp) * (double)temp : 0.0) : -INFINITY;
  auto mass = [&](int b) { return (double)s.mass[b] * (s.edge[b] / UNIT); };
  double total = 0;
  {
    double x = 0;
    for (int b = tid; b < BINS; b += NT) x += mass(b);
    total = row.sum(x);
  }
  // The lowest bin that can hold a kept token (of S1, where top_k and top_p work together), and how many tokens
  // there are from it on: at most e^(1/32) for each unit of e^x.
  double above = 0;
  int t = 0;
  if (k) t = max(0, row.cross((double)k, above, [&](int b) { return (double)s.count[b]; }));
  else if (by_p) t = max(0, row.cross(p * total, above, mass));
  if (by_m && !(k && by_p)) t = max(t, min(row.bin((float)floor_l) - 1, BINS - 1));
  double from = 0;
  for (int b = tid; b < BINS; b += NT)
    if (b >= t) from += k ? (double)s.count[b] : (double)s.mass[b] * (1.0321 / UNIT);
  from = row.sum(from);
  if (from <= LIST) {
    const int n = row.collect([&](float l, int) { return row.bin(l) >= t; });
    row.finish_list(min(n, LIST), k, p, floor_l, total, u, r);
    return;
  }
  // Many: the cuts one after the other.
  if (k) {
    const int b = row.cross((double)k, above, [&](int x) { return (double)s.count[x]; });
    if (b >= 0) cut = row.cut_in_bin(b, above, (double)k, true);
  }
  if (by_p) {
    if (k) {
      // the histogram once more (the cut's own may have taken its place), and the weight of S1
      total = row.shares(cut);
      unsigned long long b2;
      bool n2;
      row.survey(true, false, b2, n2);
      __syncthreads();
    }
    const int b = row.cross(p * total, above, mass);
    if (b >= 0) cut = row.cut_in_bin(b, above, p * total, false);
  }
  if (by_m) {
    // smallest key of a logit that is no lower
    float f = (float)floor_l;
    if ((double)f < floor_l) f = value_of(key_of(f) + 1);
    const unsigned m = min(key_of(f), (unsigned)(best >> 32));
    if (m > cut.key) cut = Cut{m, INT_MAX};
  }
  total = row.shares(cut);
  row.draw_from_shares(cut, total, u, r);
}

template <class T> void launch_t(const SampleArgs& a, hipStream_t st) { sample_kernel<T, 1024><<<a.rows, 1024, 0, st>>>(a); }

}  // namespace

void launch_sample(int dtype, const SampleArgs& a, hipStream_t st) {
  if (dtype == 0) launch_t<bf16>(a, st);
  else if (dtype == 1) launch_t<float>(a, st);
  else launch_t<f16>(a, st);
}
