// Sampling of a token per row of logits, from given random numbers:
//   z = l / T,  w = exp(z - max z),  tokens ordered by falling logit, then by rising index
//   S1 = the first top_k tokens, S2 = the shortest prefix of S1 with at least top_p of S1's weight,
//   S3 = the tokens with w >= min_p; kept are S2 and S3 together, the first token always
//   token = the first one, in the vocabulary's order, at which the kept weight summed so far exceeds u times all of it
//
// A drawn token changes where a sum crosses a border, so weights are computed and summed in 64 bits, by fixed
// orders or in integers: the same bits whatever order the waves run in.
//
// With t = 16 (l - m0) / T, m0 a reference near the row's maximum, the weight relative to m0 is
//   w = E[b] e^(x / 16),  b = t rounded,  x = t - b in [-1/2, 1/2],  E[b] = exp(b / 16)
// the second factor by 7 terms of its series (2^-47), E from a table.  (So equal logits at m0
// have the weight 1, and their sums are exact.)  The bins b are at the same time those of a histogram,
// of e^(x / 16) in units of 2^-44 (and of tokens, where top_k asks for them).  2048 bins reach from 33 nats below m0
// (2^-47 of the largest weight) to 95 above.  Five launches, the rows' parts side by side in the second and the fourth:
//   begin    m0, the largest of a row's first tokens; clears the row's histogram
//   survey   one pass over the row: the histogram and the maximum (without filters: the weights of its pieces)
//   decide   the bin at which each filter cuts
//   collect  a second pass: the tokens of the bins from there on into a list; where these would be too many those
//            of the bin of the cut alone, and the weight of each piece's higher bins
//   finish   cuts the list and draws: within the list, or in a piece, 256 tokens of it, a token
// A sixth one does whole rows in one workgroup, where the others found that they cannot: a logit that is infinite or
// more than 95 T above m0 (at T = 0.05, 4.75: the row's maximum is often that far above its first 4096 tokens'; or these all have
// a mask's finite value), or a list too long (one value tens of thousands of times).  256 rows of 126464, one value in 3161 6 higher,
// top-p: T = 0.1 57 us, 0.05 144; beginning with 5000 masked tokens, T = 1 241, else 100.
//
// What bounds it: of many rows the first pass's reads (1024 rows of 152064 fp32 with filters of every kind: 136 us, 4.6 TB/s),
// then the second pass over the pieces that can hold a kept token (59 us) and the launches beside them (59 us; 2048 such rows
// 503 us in all); of one row the six launches and cold instructions, 30 us.  One workgroup a row, as a single
// launch, took 3566 us and 330 us.  Calls split into groups of rows whose logits stay in the last-level cache for collect:
// collect is no faster, and the short launches are paid for each group (797 us against 628, before pieces were passed over).
#include <algorithm>
#include <climits>

#include "sample.h"

namespace {

constexpr int BINS = 2048, BELOW = 33 * 16;      // bins, and those below m0
// A list of every token that may be kept is no longer than FEW, unless top_k and top_p work together: the list of one bin
// and the pieces' weights take less time than long lists (4096: 2048 rows 537 us, 1024: 499 us).
constexpr int FEW = 1024;
constexpr double UNIT = 17592186044416.0;        // 2^44
constexpr int PIECE = 1024, PIECES = SAMPLE_MAX_VOCAB / PIECE;      // tokens whose weights are one sum of the row's

#define INLINE __device__ __forceinline__
#define RARE __device__ __attribute__((noinline))

// bits whose order as unsigned is that of the floats; -0 like 0
INLINE unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
INLINE float value_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
constexpr unsigned KEY_LOWEST = 0x007fffffu;     // of -infinity
constexpr float MOST = 3.4028235e38f;

typedef __attribute__((address_space(1))) unsigned long long* Units;
typedef __attribute__((address_space(1))) double* Doubles;
typedef __attribute__((address_space(1))) unsigned* Keys;

template <int NT> struct Shared {
  unsigned long long mass[BINS + 64];            // (64 places for what has no bin: a lane each)
  unsigned count[BINS + 64];
  double edge[BINS + 64];
  double seg[PIECES];                            // sums of the row's pieces, or of the waves' shares
  double redd[NT / 64];
  unsigned redu[NT / 64];
  unsigned long long first;
  double cut;
  int n, flag;
};
constexpr int ROW_NT = 1024, PART_NT = 256;      // threads of a workgroup that has a row; a part of one
template <> struct Shared<PART_NT> {
  union {                                        // (a part is surveyed with one or the other)
    unsigned long long mass[BINS + 64];
    double edge[BINS + 64];
  };
  unsigned count[BINS + 64];
  unsigned redu[PART_NT / 64];
};
template <int NT> INLINE Shared<NT>& lds() {
  __shared__ Shared<NT> s;
  return s;
}
INLINE int lane_id() { return threadIdx.x & 63; }
INLINE int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// ---- sums and maxima over the wave and the workgroup, for every thread
template <int CTRL, int ROWS> INLINE double moved(double x) {
  const long long b = __double_as_longlong(x);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((long long)hi << 32 | lo);
}
INLINE double lane_value(double x, int lane) {
  const long long b = __double_as_longlong(x);
  return __longlong_as_double((long long)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 |
                              (unsigned)__builtin_amdgcn_readlane((int)b, lane));
}
// inclusive sums over the lanes: row_shr 1, 2, 4, 8, row_bcast 15, 31
INLINE double wave_scan64(double x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);
  x += moved<0x143, 0xc>(x);
  return x;
}
INLINE double wave_sum64(double x) { return lane_value(wave_scan64(x), 63); }
INLINE unsigned wave_max32(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
// inclusive sums in thread order
template <int NT> INLINE double scan_all(double x, double& all) {
  auto& s = lds<NT>();
  const int lane = lane_id(), w = wave_id();
  x = wave_scan64(x);
  __syncthreads();
  if (lane == 63) s.redd[w] = x;
  __syncthreads();
  const double y = wave_scan64(lane < NT / 64 ? s.redd[lane] : 0.0);
  all = lane_value(y, 63);
  return x + (w ? lane_value(y, w - 1) : 0.0);
}
template <int NT> INLINE double sum_all(double x) {
  double all;
  scan_all<NT>(x, all);
  return all;
}
template <int NT> INLINE unsigned max_all(unsigned x) {
  auto& s = lds<NT>();
  x = wave_max32(x);
  __syncthreads();
  if (lane_id() == 0) s.redu[wave_id()] = x;
  __syncthreads();
  return wave_max32(lane_id() < NT / 64 ? s.redu[lane_id()] : 0);
}

// ---- weights
// w relative to m0 is edge[bin] * e^(x / 16)
struct Place {
  int bin;       // outside [0, BINS): below every bin, or above
  double x;
};
INLINE bool in_bins(const Place& p) { return (unsigned)p.bin < (unsigned)BINS; }
// With y = x / 16, c + y + y^2 / 2 + ... + y^6 / 720: e^y for c = 1, off by 2^-47
INLINE double series(double x, double c) {
  double e = fma(x, 0x1p-24 / 720, 0x1p-20 / 120);
  e = fma(e, x, 0x1p-16 / 24);
  e = fma(e, x, 0x1p-12 / 6);
  e = fma(e, x, 0x1p-8 / 2);
  e = fma(e, x, 0x1p-4);
  return fma(e, x, c);
}
// that in units of 2^-44: the last bits of 256 + e^y
INLINE unsigned long long units(double x) {
  return (unsigned long long)__double_as_longlong(series(x, 257.0)) - 0x4070000000000000ull;
}
INLINE double scale_of(float temp) { return fmax(16.0 / (double)temp, 0x1p-900); }      // (-infinity times it is -infinity)
// the bin, or a place of the lane's own behind the bins
INLINE unsigned bin_or_lane(const Place& p, int lane) { return min((unsigned)p.bin, (unsigned)(BINS + lane)); }

// x, the same in every lane, in a scalar register
INLINE double uniform(double x) { return lane_value(x, 0); }

typedef unsigned u32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x4a2 __attribute__((ext_vector_type(4), aligned(2)));

// A row, and how its logits become weights.
template <class T> struct View {
  static constexpr int N = 16 / sizeof(T);
  typedef const __attribute__((address_space(1))) T* Ptr;
  using Vec = std::conditional_t<sizeof(T) == 4, u32x4a4, u32x4a2>;
  typedef const __attribute__((address_space(1))) Vec* VecPtr;
  Ptr row;
  int V, share, exclude;     // share: a wave has the tokens wave share .. + share - 1
  bool inf;                  // the row's maximum is infinite: its tokens alone, alike
  double m0, scale;          // scale = 16 / T

  INLINE float logit(float x, int i) const {
    if (i == exclude) return -INFINITY;
    return inf ? (x == INFINITY ? 0.f : x != x ? x : -INFINITY) : x;
  }
  INLINE Place place(float l) const {
    const double t = fma((double)l - m0, scale, (double)BELOW), f = rint(t);
    Place p;
    p.x = t - f;
    asm("v_cvt_i32_f64 %0, %1" : "=v"(p.bin) : "v"(f));      // (saturates, where a cast would be undefined)
    return p;
  }
  // logits surely below and surely above bin b
  INLINE float below(int b) const { return beyond(b - 1, -0x1p-20); }
  INLINE float above(int b) const { return beyond(b + 1, 0x1p-20); }
  INLINE float beyond(int b, double by) const {
    const double d = m0 + (b - BELOW) / scale;
    return fminf(fmaxf((float)(d + fabs(d) * by), -MOST), MOST);
  }
};
template <int NT, class T> INLINE double weight(const View<T>& v, float l) {
  const Place p = v.place(l);
  return in_bins(p) ? lds<NT>().edge[p.bin] * series(p.x, 1.0) : 0.0;
}
// the greater one, of numbers (as an instruction: the compiler would first make a quiet NaN of a signalling one)
INLINE float at_least(float x, float low) {
  asm("v_max_f32 %0, %0, %1" : "+v"(x) : "v"(low));
  return x;
}

// f(logits, indexes) for the tokens [i0, i1), by the calling wave, 8 a lane at a time; i0 and i1 are the wave's.
// A half's next loads are on their way while the other half is worked on.
// after(i) follows each piece of 1024, from i on, and next(i) says where the next one is.
template <class T, class F, class G, class X> INLINE void tokens(const View<T>& v, int i0, int i1, F&& f, G&& after, X&& next) {
  constexpr int N = View<T>::N, H = 8, P = H / N, HALF = 64 * H;
  const int lane = lane_id();
  i1 = min(i1, v.V);
  typename View<T>::Vec x[2][P];
  auto fetch = [&](int half, int i) __attribute__((always_inline)) {
    if (i >= i1 || v.V < N) return;
#pragma unroll
    for (int p = 0; p < P; ++p) x[half][p] = *(typename View<T>::VecPtr)(v.row + min(i + (p * 64 + lane) * N, v.V - N));
  };
  fetch(0, i0);
  fetch(1, i0 + HALF);
#pragma unroll 1
  for (int i = i0; i < i1;) {
    const int n = next(i);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int b = i + half * HALF;
      if (half && b >= i1) break;
      float l[H];
      auto index = [&](int e) __attribute__((always_inline)) { return b + (e / N * 64 + lane) * N + e % N; };
#pragma unroll
      for (int e = 0; e < H; ++e) {
        T y[N];
        __builtin_memcpy(y, &x[half][e / N], 16);
        l[e] = to_f32(y[e % N]);
      }
      // past the end, or with a token that is not what its logit says: one by one
      if (v.inf | (b + HALF > i1) | ((unsigned)(v.exclude - b) < (unsigned)HALF)) {
#pragma unroll
        for (int e = 0; e < H; ++e) l[e] = to_f32(v.row[min(index(e), v.V - 1)]);
#pragma unroll
        for (int e = 0; e < H; ++e) l[e] = index(e) < i1 ? v.logit(l[e], index(e)) : -INFINITY;
      }
      f(l, index);
      fetch(half, n + half * HALF);
    }
    after(i);
    i = n;
  }
}
template <class T, class F> INLINE void tokens(const View<T>& v, int i0, int i1, F&& f) {
  tokens(v, i0, i1, f, [](int) {}, [](int i) { return i + PIECE; });
}
template <class T, class F> INLINE void all_tokens(const View<T>& v, F&& f) {
  const int w = wave_id();
  tokens(v, w * v.share, (w + 1) * v.share, f);
}
// the largest, or a NaN where there is one
template <int M> INLINE float largest(const float (&l)[M]) {
  float m = l[0];
#pragma unroll
  for (int e = 1; e < M; ++e) m = __builtin_elementwise_maximum(m, l[e]);
  return m;
}

// ---- the first pass
// Histogram of the wave's tokens [i0, i1) about m0 (counts, masses) and the keys of their pieces' maxima into tops, or the
// weights of their pieces into seg; the key of their maximum, all ones where there is a NaN.
template <int MODE, int NT, class T> INLINE unsigned survey_as(const View<T>& v, int i0, int i1, float low, Keys tops, Doubles seg) {
  constexpr bool COUNTS = MODE & 1, MASSES = MODE & 2;
  auto& s = lds<NT>();
  const int lane = lane_id();
  double x = 0;
  float top = -INFINITY;
  unsigned best = 0;
  tokens(v, i0, i1, [&](auto& l, auto) __attribute__((always_inline)) {
    constexpr int M = sizeof(l) / 4;
    const float most = largest(l);
    top = __builtin_elementwise_maximum(top, most);
    if (!__ballot(most >= low)) return;               // all of them below the bins
    Place p[M];
#pragma unroll
    for (int e = 0; e < M; ++e) p[e] = v.place(l[e]);
#pragma unroll
    for (int e = 0; e < M; ++e) {
      const unsigned b = bin_or_lane(p[e], lane);
      if (COUNTS) atomicAdd(&s.count[b], 1u);
      if (MASSES) atomicAdd(&s.mass[b], units(p[e].x));
      if (!MODE) x += s.edge[b] * series(in_bins(p[e]) ? p[e].x : 0.0, 1.0);
    }
  }, [&](int i) __attribute__((always_inline)) {
    const unsigned t = wave_max32(top != top ? 0xffffffffu : key_of(top));
    best = max(best, t);
    top = -INFINITY;
    if (MODE) {
      if (lane == 0 && tops) tops[i / PIECE] = t;
      return;
    }
    x = wave_sum64(x);
    if (lane == 0) seg[i / PIECE] = x;
    x = 0;
  }, [](int i) { return i + PIECE; });
  return best;
}
// That of all the workgroup's tokens.
template <int NT, class T> INLINE unsigned survey(const View<T>& v, bool masses, bool counts, int i0, int i1, Keys tops, Doubles seg) {
  const float low = v.below(0);
  return max_all<NT>(masses && counts ? survey_as<3, NT>(v, i0, i1, low, tops, seg)
                     : masses         ? survey_as<2, NT>(v, i0, i1, low, tops, seg)
                     : counts         ? survey_as<1, NT>(v, i0, i1, low, tops, seg)
                     : seg            ? survey_as<0, NT>(v, i0, i1, low, tops, seg)
                                      : 0);
}

// The largest logit of the wave's tokens [i0, i1) with its first index (key above, ~index below), or all ones for a NaN.
template <class T> INLINE unsigned long long first_token(const View<T>& v, int i0, int i1) {
  unsigned long long top = 0;
  tokens(v, i0, i1, [&](auto& l, auto index) __attribute__((always_inline)) {
    constexpr int M = sizeof(l) / 4;
#pragma unroll
    for (int e = 0; e < M; ++e) {
      const unsigned long long k = l[e] != l[e] ? ~0ull : (unsigned long long)key_of(l[e]) << 32 | (unsigned)~index(e);
      top = max(top, k);
    }
  });
  return top;
}

// ---- the second pass
// The wave's tokens [i0, i1) of bin b, or with ALL those of every bin from b on, to put(~key, index).  Without ALL the
// weights of the pieces' higher bins go into seg.  Pieces whose maximum (tops) is lower are not read: 64 of them at most.
// (A logit below `low` is raised to it for a place that is finite.  At temperatures from 1e37 on, where `low` ends at the
// lowest float, that place may be in bin b or above it: so the logit is looked at, too.)
template <bool ALL, int NT, class T, class F> INLINE void collect(const View<T>& v, int b, int i0, int i1, Keys tops, Doubles seg, F&& put) {
  auto& s = lds<NT>();
  const int lane = lane_id(), mine = i0 + lane * PIECE;
  const float low = v.below(b);
  const bool in = mine < min(i1, v.V), high = in && tops[in ? mine / PIECE : 0] >= key_of(low);
  if (!ALL && in && !high) seg[mine / PIECE] = 0;
  unsigned long long left = __ballot(high);
  auto piece = [&] { return left ? i0 + (__ffsll(left) - 1) * PIECE : 1 << 30; };
  double x = 0;
  tokens(v, piece(), i1, [&](auto& l, auto index) __attribute__((always_inline)) {
    constexpr int M = sizeof(l) / 4;
    if (!__ballot(largest(l) >= low)) return;
    Place p[M];
    if (!ALL) {
#pragma unroll
      for (int e = 0; e < M; ++e) p[e] = v.place(at_least(l[e], low));
#pragma unroll
      for (int e = 0; e < M; ++e) x += s.edge[(p[e].bin > b) & (l[e] >= low) ? p[e].bin : BINS] * series(p[e].x, 1.0);
    }
#pragma unroll
    for (int e = 0; e < M; ++e) {
      if (l[e] >= low && (ALL || (p[e].bin == b && b >= 0))) {
        if (ALL && v.place(l[e]).bin < b) continue;
        put((unsigned long long)~key_of(l[e]) << 32 | (unsigned)index(e));
      }
    }
  }, [&](int i) __attribute__((always_inline)) {
    if (ALL) return;
    x = wave_sum64(x);
    if (lane == 0) seg[i / PIECE] = x;
    x = 0;
  }, [&](int) __attribute__((always_inline)) {
    left &= left - 1;
    return piece();
  });
}
INLINE float logit_of(unsigned long long e) { return value_of(~(unsigned)(e >> 32)); }

// Tokens that are held in memory: ~key, index, which rises in the order of the tokens; and their weights, in
// units of 2^-49 of the largest there can be (so that all of them are below 2^63).
struct List {
  Units e, w;
  int n;
};

INLINE void write(const SampleArgs& a, int r, int token, float logp) {
  a.token[r] = token;
  if (a.logp) a.logp[r] = logp;
}

// ---- cuts
// The bin, from the highest on, at whose end the sum over the bins reaches `target` (strict: exceeds it), and the sum above
// it; -1 where it does not.  The sum is that of the counts (unit 0), of the masses in `unit`, or (unit < 0) in those of
// the bins' edges.  A wave's or thread's end and the next one's start are sums of other groupings and may differ in their last
// bits.  So the crossing is in the first wave of any weight whose end reaches the target, and there at the first such thread, then
// bin, or the last one of any weight if the end is reached at none: one thread's, whatever the rounding.
template <int NT> INLINE int cross(double target, double unit, double& above, bool strict = false) {
  constexpr int E = BINS / NT;
  auto& s = lds<NT>();
  const int lane = lane_id(), w = wave_id();
  auto reached = [&](double y) { return strict ? y > target : y >= target; };
  double x[E], t = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int b = BINS - 1 - (threadIdx.x * E + e);
    x[e] = unit == 0 ? (double)s.count[b] : (double)s.mass[b] * (unit < 0 ? s.edge[b] * (1 / UNIT) : unit);
    t += x[e];
  }
  const double upto = wave_scan64(t);
  if (lane == 63) s.redd[w] = upto;
  __syncthreads();
  const double wave = lane < NT / 64 ? s.redd[lane] : 0.0, ends = wave_scan64(wave);
  const unsigned long long waves = __ballot(wave > 0 && reached(ends));
  if (waves ? w == __ffsll(waves) - 1 : w == 0) {
    double y = upto + (w ? lane_value(ends, w - 1) : 0.0);
    const unsigned long long any = __ballot(t > 0), hit = __ballot(t > 0 && reached(y));
    if (lane == (hit ? __ffsll(hit) - 1 : any ? 63 - __clzll((long long)any) : 0)) {
      y -= t;
      double cut = y;
      int at = 0;
      bool open = true;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool here = open && x[e] > 0;
        at = here ? e : at;
        cut = here ? y : cut;
        y += x[e];
        open = open && !(here && reached(y));
      }
      s.cut = cut;
      s.flag = waves ? BINS - 1 - (threadIdx.x * E + at) : -1;
    }
  }
  __syncthreads();
  above = s.cut;
  return s.flag;
}
// the lowest bin that has a token
template <int NT> RARE int lowest() {
  auto& s = lds<NT>();
  unsigned low = 0;
  for (int j = threadIdx.x; j < BINS; j += NT)
    if (s.count[j]) low = max(low, (unsigned)(BINS - j));
  return BINS - (int)max_all<NT>(low);
}

// What is kept: the tokens of greater keys, and of this one those up to index `last`.
struct Cut {
  unsigned key;
  int last;
};
INLINE Cut everything() { return Cut{KEY_LOWEST + 1, INT_MAX}; }      // (the lowest finite value's tokens among it)

// clears the parts of the keys lo .. hi; how far a key's distance from lo is shifted to be its part
template <int NT> INLINE int clear_parts(unsigned lo, unsigned hi) {
  auto& s = lds<NT>();
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += NT) s.mass[i] = s.count[i] = 0;
  __syncthreads();
  return max(0, 32 - __clz((int)(hi - lo)) - 11);
}
// The part of the keys lo .. hi in which `target` is reached: narrows lo and hi to it and raises `above` by what is
// above it.  The parts are in s.count and, unless by_count, s.mass, in `unit`.  Returns its tokens.
template <int NT> INLINE int narrow(unsigned& lo, unsigned& hi, int shift, double& above, double target, bool by_count, double unit) {
  auto& s = lds<NT>();
  double more;
  int i = cross<NT>(target - above, by_count ? 0.0 : unit, more);
  if (i < 0) {                         // not reached, by rounding: the last of them all
    i = lowest<NT>();
    more = -INFINITY;
  }
  above += more;
  lo += (unsigned)i << shift;
  hi = min(hi, lo + (1u << shift) - 1);
  const int n = s.count[i];
  __syncthreads();
  return n;
}

// f(element, weight) for the list's tokens: four of a thread are on their way together.
template <int NT, class F> INLINE void each_of(const List& q, F&& f) {
#pragma unroll 1
  for (int i = threadIdx.x; i < q.n; i += 4 * NT) {
    unsigned long long e[4], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = min(i + j * NT, q.n - 1);
      e[j] = q.e[at];
      w[j] = q.w[at];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * NT < q.n) f(e[j], w[j], i + j * NT);
  }
}
// Weights of the list's tokens, in units of 2^-49 of w1, which none exceeds; returns the unit.
template <int NT, class T> INLINE double list_weights(const View<T>& v, const List& q, double w1) {
  const double scale = 0x1p49 / w1;
  each_of<NT>(q, [&](unsigned long long e, unsigned long long, int i) { q.w[i] = (unsigned long long)rint(weight<NT>(v, logit_of(e)) * scale); });
  __syncthreads();
  return w1 * 0x1p-49;
}

// The cut within the list, of keys lo .. hi: its element.  What is above the list amounts to `above`, the cut is
// where `target` is reached; by_count: tokens are counted, else their weights summed.
template <int NT> INLINE unsigned long long cut_in_list(const List& q, unsigned lo, unsigned hi, double above, double target, bool by_count, double unit) {
  auto& s = lds<NT>();
  const int tid = threadIdx.x;
  // narrower and narrower, to one token or one value
  int k = q.n;
#pragma unroll 1
  while (k > 1 && lo < hi) {
    const int shift = clear_parts<NT>(lo, hi);
    each_of<NT>(q, [&](unsigned long long e, unsigned long long w, int) {
      const unsigned key = ~(unsigned)(e >> 32);
      if (key >= lo && key <= hi) {
        atomicAdd(&s.count[(key - lo) >> shift], 1u);
        if (!by_count) atomicAdd(&s.mass[(key - lo) >> shift], w);
      }
    });
    k = narrow<NT>(lo, hi, shift, above, target, by_count, unit);
  }
  // of those left, all of one value, the want-th by index: in parts of the row, the first ones highest
  if (tid == 0) s.n = 0;
  int part = 0, shift = 0, want = 1;
  if (k > 1) {
    double w = 1;
    if (!by_count) {
      each_of<NT>(q, [&](unsigned long long e, unsigned long long w, int) {
        if (~(unsigned)(e >> 32) == lo) s.first = w;
      });
      __syncthreads();
      w = (double)s.first * unit;
    }
    want = (int)fmin(fmax(1.0, ceil((target - above) / w)), (double)k);
    shift = clear_parts<NT>(0u, SAMPLE_MAX_VOCAB - 1);
    each_of<NT>(q, [&](unsigned long long e, unsigned long long, int) {
      if (~(unsigned)(e >> 32) == lo) atomicAdd(&s.count[BINS - 1 - ((unsigned)e >> shift)], 1u);
    });
    double before;
    part = BINS - 1 - cross<NT>((double)want, 0.0, before);
    want -= (int)before;
  }
  __syncthreads();
  each_of<NT>(q, [&](unsigned long long e, unsigned long long, int) {
    const unsigned key = ~(unsigned)(e >> 32);
    if (key >= lo && key <= hi && (k == 1 || (unsigned)e >> shift == (unsigned)part)) s.mass[atomicAdd(&s.n, 1)] = e;
  });
  __syncthreads();
  const int m = s.n;
  if (tid < m) {
    int rank = 1;
    for (int j = 0; j < m; ++j) rank += s.mass[j] < s.mass[tid];
    if (rank == want) s.first = s.mass[tid];
  }
  __syncthreads();
  const unsigned long long e = s.first;
  __syncthreads();
  return e;
}
// the sum of f(element, weight)
template <int NT, class F> INLINE unsigned long long sum_units(const List& q, F&& f) {
  auto& s = lds<NT>();
  unsigned long long x = 0;
  __syncthreads();
  if (threadIdx.x == 0) s.first = 0;
  __syncthreads();
  each_of<NT>(q, [&](unsigned long long e, unsigned long long w, int) { x += f(e, w); });
  if (x) atomicAdd(&s.first, x);
  __syncthreads();
  x = s.first;
  __syncthreads();
  return x;
}
// the last element of the order whose logit is no lower than floor_l, and at least the best one
INLINE unsigned long long last_of(double floor_l, unsigned best) {
  float f = (float)floor_l;
  if ((double)f < floor_l) f = value_of(key_of(f) + 1);
  return (unsigned long long)~min(key_of(f), best) << 32 | 0xffffffffu;
}

// The list holds the first tokens of the order, those of the bins from t on: filters and draw among them.
// mass1: weight of S1, where k is 0; best: the key of the largest logit.
template <int NT, class T>
INLINE void finish_list(const SampleArgs& a, const View<T>& v, const List& q, int k, bool by_p, double p, double floor_l, double mass1, unsigned best, int t, double u, int r) {
  auto& s = lds<NT>();
  const int tid = threadIdx.x;
  const double unit = list_weights<NT>(v, q, weight<NT>(v, value_of(best)));
  const unsigned lo = key_of(v.below(t));
  unsigned long long last = ~0ull;             // the last kept element of the list
#pragma unroll 1
  for (int by = 0; by < 2; ++by) {             // top_k, then top_p
    if (by == 0 ? !(k > 0 && k < q.n) : !by_p) continue;
    double target = (double)k;
    if (by == 1) target = p * (k > 0 ? (double)sum_units<NT>(q, [&](unsigned long long e, unsigned long long w) { return e <= last ? w : 0; }) * unit : mass1);
    last = min(last, cut_in_list<NT>(q, lo, best, 0.0, target, by == 0, unit));
  }
  if (floor_l > -INFINITY) last = min(last, last_of(floor_l, best));
  // in the vocabulary's order: parts of the row, the first ones highest
  const int shift = clear_parts<NT>(0u, (unsigned)(v.V - 1));
  const double total = (double)sum_units<NT>(q, [&](unsigned long long e, unsigned long long w) {
    const unsigned long long x = e <= last ? w : 0;
    const int part = BINS - 1 - (int)((unsigned)e >> shift);
    if (x) {
      atomicAdd(&s.mass[part], x);
      atomicAdd(&s.count[part], 1u);
    }
    return x;
  });
  const double target = u * total;
  if (tid == 0) s.n = 0;
  double before;
  int part = cross<NT>(target, 1.0, before, true);
  if (part < 0) {                              // u near one and the sums' rounding: the last part of any weight
    part = lowest<NT>();
    before = -1;
  }
  // the part's tokens (no more than the row has in a part), by one wave
  each_of<NT>(q, [&](unsigned long long e, unsigned long long w, int i) {
    if (e <= last && w && BINS - 1 - (int)((unsigned)e >> shift) == part) s.count[atomicAdd(&s.n, 1)] = i;
  });
  __syncthreads();
  if (wave_id() != 0) return;
  const int m = s.n;
  unsigned hit = 0xffffffffu, end = 0;
#pragma unroll 1
  for (int j = lane_id(); j < m; j += 64) {
    const unsigned at = (unsigned)q.e[s.count[j]];
    unsigned long long upto = 0;
    for (int o = 0; o < m; ++o) upto += (unsigned)q.e[s.count[o]] <= at ? q.w[s.count[o]] : 0;
    if (before >= 0 && before + (double)upto > target) hit = min(hit, at);
    end = max(end, at);
  }
  hit = ~wave_max32(~hit);
  end = wave_max32(end);
  const unsigned token = hit != 0xffffffffu ? hit : end;
#pragma unroll 1
  for (int j = lane_id(); j < m; j += 64) {
    const unsigned long long e = q.e[s.count[j]];
    if ((unsigned)e == token) write(a, r, (int)token, (float)log(weight<NT>(v, logit_of(e)) / (total * unit)));
  }
}

// Sums of the kept weights of the waves' parts of the tokens [i0, i1), in s.seg.
template <int NT, class T> INLINE void sum_parts(const View<T>& v, const Cut& c, int i0, int i1, int part) {
  auto& s = lds<NT>();
  const int lane = lane_id(), w = wave_id();
  const float at = value_of(max(c.key, KEY_LOWEST + 1));
  double x = 0;
  tokens(v, i0 + w * part, min(i0 + (w + 1) * part, i1), [&](auto& l, auto index) __attribute__((always_inline)) {
    constexpr int M = sizeof(l) / 4;
    if (!__ballot(largest(l) >= at)) return;
    Place p[M];
#pragma unroll
    for (int e = 0; e < M; ++e) p[e] = v.place(at_least(l[e], at));
#pragma unroll
    for (int e = 0; e < M; ++e) {
      const bool in = (l[e] > at) | ((l[e] == at) & (index(e) <= c.last));
      x += s.edge[in ? bin_or_lane(p[e], lane) : BINS] * series(p[e].x, 1.0);
    }
  });
  x = wave_sum64(x);
  __syncthreads();
  if (lane == 0) s.seg[w] = x;
  __syncthreads();
}

// Smallest key of a logit whose bin is at least b: near m0 + (b - BELOW - 1/2) / scale.
template <class T> INLINE unsigned first_key(const View<T>& v, int b) {
  auto reaches = [&](unsigned k) { return v.place(value_of(k)).bin >= b; };
  const double x = fmin(fmax(v.m0 + (b - BELOW - 0.5) / v.scale, (double)-MOST), (double)MOST);
  unsigned k = min(max(key_of((float)x), KEY_LOWEST + 1), key_of(INFINITY)), step = 1;
  // a few steps away, unless the bins are narrower than the floats' own steps or wider than them all
  const bool down = reaches(k);
  auto room = [&] { return down ? k - (KEY_LOWEST + 1) >= step : key_of(INFINITY) - k > step; };
  auto next = [&] { return down ? k - step : k + step; };
  bool rising = true;
#pragma unroll 1
  while (step) {
    if (room() && reaches(next()) == down) {
      k = next();
      if (rising) step *= 2;
    } else {
      rising = false;
      step /= 2;
    }
  }
  return down ? k : k + 1;
}

// Index of the n-th token of this key.
template <int NT, class T> INLINE int nth(const View<T>& v, unsigned key, int n) {
  auto& s = lds<NT>();
  const int lane = lane_id(), w = wave_id();
  int c = 0;
  all_tokens(v, [&](auto& l, auto) __attribute__((always_inline)) {
    constexpr int M = sizeof(l) / 4;
#pragma unroll
    for (int e = 0; e < M; ++e) c += key_of(l[e]) == key;
  });
  for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o, 64);
  __syncthreads();
  if (lane == 0) s.redu[w] = c;
  __syncthreads();
  int at = 0;
  while (at < NT / 64 - 1 && n > (int)s.redu[at]) n -= (int)s.redu[at++];
  __syncthreads();
  if (w == 0) {
    const int p1 = min((at + 1) * v.share, v.V);
    int res = p1 - 1;
#pragma unroll 1
    for (int p = at * v.share; p < p1; p += 64) {
      const int i = p + lane, j = min(i, v.V - 1);
      const unsigned long long m = __ballot(i < p1 && key_of(v.logit(to_f32(v.row[j]), j)) == key);
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
// The cut within bin b: the tokens of higher bins amount to `above`, the cut is where `target` is reached.  In the
// row, by one workgroup, to one value.
template <int NT, class T> INLINE Cut cut_in_row(const View<T>& v, int b, double above, double target, bool by_count) {
  auto& s = lds<NT>();
  unsigned lo = first_key(v, b), hi = b + 1 < BINS ? first_key(v, b + 1) - 1 : key_of(INFINITY);
  const double unit = s.edge[b] * (1 / UNIT);
  int k = 1;
#pragma unroll 1
  for (;;) {
    const int shift = clear_parts<NT>(lo, hi);
    const float from = value_of(lo);
    all_tokens(v, [&](auto& l, auto) __attribute__((always_inline)) {
      constexpr int M = sizeof(l) / 4;
      if (!__ballot(largest(l) >= from)) return;
#pragma unroll
      for (int e = 0; e < M; ++e) {
        const unsigned key = key_of(l[e]);
        if (key >= lo && key <= hi) {
          atomicAdd(&s.count[(key - lo) >> shift], 1u);
          if (!by_count) atomicAdd(&s.mass[(key - lo) >> shift], units(v.place(l[e]).x));
        }
      }
    });
    k = narrow<NT>(lo, hi, shift, above, target, by_count, unit);
    if (lo >= hi) break;
  }
  const double each = by_count ? 1.0 : weight<NT>(v, value_of(lo));
  return Cut{lo, nth<NT>(v, lo, (int)fmin(fmax(1.0, ceil((target - above) / each)), (double)k))};
}

// Of s.seg's first n: the one at which what is before and the sums so far exceed target, or the last with any
// weight; what is before it.
template <int NT> INLINE int descend(int n, double target, double& before) {
  const int lane = lane_id();
  double y = before;
  int at = 0;
#pragma unroll 1
  for (int i = 0; i < n; i += 64) {
    const double x = i + lane < n ? lds<NT>().seg[i + lane] : 0.0, z = y + wave_scan64(x);
    const unsigned long long hit = __ballot(x > 0 && z > target), pos = __ballot(x > 0);
    if (hit | pos) {
      const int j = hit ? __ffsll(hit) - 1 : 63 - __clzll((long long)pos);
      at = i + j;
      before = lane_value(z - x, j);
    }
    if (hit) break;
    y = lane_value(z, 63);
  }
  return at;
}
template <int NT> INLINE double seg_total(int n) {
  double x = 0;
  for (int i = lane_id(); i < n; i += 64) x += lds<NT>().seg[i];
  return wave_sum64(x);
}

// The token at which the kept weight exceeds u times all of it, from the sums of the row's n parts in s.seg: descend into a
// part, then into a wave's share of it, and so on, then token by token.
template <int NT, class T> INLINE void draw(const SampleArgs& a, const View<T>& v, const Cut& c, int n, int part, double u, int r) {
  constexpr int NW = NT / 64;
  const int lane = lane_id();
  const double total = seg_total<NT>(n), target = u * total;
  double before = 0;
  int i0 = descend<NT>(n, target, before) * part;
#pragma unroll 1
  while (part > 256) {
    const int i1 = i0 + part;
    part = (part / NW + 255) / 256 * 256;
    __syncthreads();
    sum_parts<NT>(v, c, i0, i1, part);
    i0 += descend<NT>(NW, target, before) * part;
  }
  const int p1 = min(i0 + part, v.V);
  if (wave_id() != 0) return;
  // one wave: 256 tokens at a time, four of a lane
  int token = -1;
  double wt = 0;
#pragma unroll 1
  for (int p = i0; p < p1; p += 256) {
    double x[4], y = 0;
    float l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) l[e] = to_f32(v.row[min(p + lane * 4 + e, v.V - 1)]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = p + lane * 4 + e;
      l[e] = i < p1 ? v.logit(l[e], i) : -INFINITY;
      const unsigned k = key_of(l[e]);
      x[e] = k > c.key || (k == c.key && i <= c.last) ? weight<NT>(v, l[e]) : 0.0;
      y += x[e];
    }
    const double z = wave_scan64(y);
    // the first lane at whose end the target is exceeded, in it the first such token of any weight
    const unsigned long long hit = __ballot(y > 0 && before + z > target), pos = __ballot(y > 0);
    if (hit | pos) {           // (not reached, by rounding: the last token of any weight)
      const int k = hit ? __ffsll(hit) - 1 : 63 - __clzll((long long)pos);
      double at = before + z - y, w = 0;
      int mine = 0;
      bool found = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        at += x[e];
        if (x[e] > 0 && !found) mine = e, w = x[e], found = hit && at > target;
      }
      token = p + k * 4 + __builtin_amdgcn_readlane(mine, k);
      wt = lane_value(w, k);
    }
    if (hit) break;
    before += lane_value(z, 63);
  }
  if (lane == 0) write(a, r, token, (float)log(wt / total));
}

// ---- the launches
enum Mode { DONE, ONE, PLAIN, FILTERS, ALL, CUT };
// A row between the launches.
struct RowState {
  double m0, scale, total, above, target, floor_l;
  unsigned long long first;     // ONE: the first token
  unsigned best;                // the key of the maximum, all ones for a NaN
  int mode, k, bin, n;          // n: tokens of the list
  int by_k, by_p, by_m;         // the cut's bin is that of top_k, of top_p, of min_p
};
constexpr int DECIDE_NT = 512;      // (finish: two such workgroups fit a CU, where one of 1024 would alone: 1024 rows 50 -> 36 us)
constexpr int LISTED = 16384, PART_LIST = 1024;      // a list's tokens in memory, and a part's of it in LDS

struct Space {
  RowState* row;
  unsigned long long* mass;     // [rows][BINS]
  unsigned* count;              // [rows][BINS]
  double* seg;                  // [rows][PIECES]
  unsigned* top;                // [rows][PIECES]: keys of the pieces' maxima
  double* edge;                 // [BINS]
  unsigned long long *e, *w;    // [rows][LISTED]
  int* whole;                   // how many rows are left to sample_whole, and which
};
struct Call {
  SampleArgs a;
  Space s;
  int row0, part, parts;        // the group's first row; a part's tokens, and how many there are
};
INLINE void leave_whole(const Space& s, int i) { s.whole[1 + atomicAdd(&s.whole[0], 1)] = i; }
struct Wants {
  double p, mp, u;
  float temp;
  int k;
  bool one, by_k, by_p, by_m;
};
INLINE Wants wants(const SampleArgs& a, int r) {
  Wants w;
  w.temp = a.temperature ? a.temperature[r] : 1.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  w.p = a.top_p ? (double)a.top_p[r] : 1.0;
  w.mp = a.min_p ? (double)a.min_p[r] : 0.0;
  const float u = a.u[r];
  w.u = u > 0.f ? (double)u : 0.0;
  w.by_k = k > 0 && k < a.vocab;
  w.by_p = w.p < 1;
  w.by_m = w.mp > 0;
  w.k = w.by_k ? k : 0;
  w.one = !(w.temp > 0.f) || w.p <= 0 || w.mp > 1;       // the first token of the order alone
  return w;
}
template <class T> INLINE View<T> view_of(const SampleArgs& a, int r, double m0, double scale) {
  View<T> v;
  v.row = (typename View<T>::Ptr)((const T*)a.logits + (size_t)r * a.ld);
  v.V = a.vocab;
  v.share = 0;
  v.exclude = a.exclude;
  v.inf = false;
  v.m0 = uniform(m0);
  v.scale = uniform(scale);
  return v;
}
template <int NT> INLINE void load_edges(const Call& c) {
  auto& s = lds<NT>();
  for (int i = threadIdx.x; i < BINS + 64; i += NT) s.edge[i] = i < BINS ? c.s.edge[i] : 0.0;
}

template <class T> __global__ __launch_bounds__(PART_NT) void sample_begin(Call c, int rows) {
  constexpr int NT = PART_NT;
  const int tid = threadIdx.x, i = blockIdx.x;
  if (i >= rows) {              // the last workgroups: the edges
    const int b = (i - rows) * NT + tid;
    c.s.edge[b] = exp((b - BELOW) / 16.0);
    if (b == 0) c.s.whole[0] = 0;
    return;
  }
  const int r = c.row0 + i;
  const Wants w = wants(c.a, r);
  const View<T> v = view_of<T>(c.a, r, 0.0, 0.0);
  if (!w.one && (w.by_k || w.by_p || w.by_m))
    for (int b = tid; b < BINS; b += NT) {
      c.s.mass[(size_t)i * BINS + b] = 0;
      c.s.count[(size_t)i * BINS + b] = 0;
    }
  // the reference: the maximum of the first 4096 tokens (or of the next ones that are not all masked), 0 if there are none
  unsigned top = KEY_LOWEST;
#pragma unroll 1
  for (int i0 = 0; i0 < v.V && top == KEY_LOWEST; i0 += 16 * NT) {
    float l[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) l[e] = to_f32(v.row[min(i0 + e * NT + tid, v.V - 1)]);      // (past the end the last one)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = v.logit(l[e], min(i0 + e * NT + tid, v.V - 1));
      if (x < INFINITY) top = max(top, key_of(x));
    }
    top = max_all<NT>(top);
  }
  if (tid) return;
  RowState& st = c.s.row[i];
  st.m0 = top > KEY_LOWEST ? (double)value_of(top) : 0.0;
  st.scale = scale_of(w.temp);
  st.first = 0;
  st.best = 0;
  st.n = 0;
  st.mode = w.one ? ONE : w.by_k || w.by_p || w.by_m ? FILTERS : PLAIN;
}

template <class T> __global__ __launch_bounds__(PART_NT) void sample_survey(Call c) {
  constexpr int NT = PART_NT;
  auto& s = lds<NT>();
  const int tid = threadIdx.x, i = blockIdx.y;
  RowState& st = c.s.row[i];
  const int mode = st.mode, share = c.part / (NT / 64), i0 = blockIdx.x * c.part + wave_id() * share;
  const View<T> v = view_of<T>(c.a, c.row0 + i, st.m0, st.scale);
  if (mode == ONE) {
    unsigned long long top = first_token(v, i0, i0 + share);
    for (int o = 32; o; o >>= 1) top = max(top, (unsigned long long)__shfl_xor(top, o, 64));
    if (lane_id() == 0) atomicMax(&st.first, top);
    return;
  }
  const Wants w = wants(c.a, c.row0 + i);
  const bool masses = mode == FILTERS && (w.by_p || (w.by_m && !w.by_k)), counts = mode == FILTERS && w.by_k;
  if (mode == PLAIN) {
    load_edges<NT>(c);
  } else {
    for (int b = tid; b < BINS; b += NT) {
      s.mass[b] = 0;
      s.count[b] = 0;
    }
  }
  __syncthreads();
  const unsigned best = survey<NT>(v, masses, counts, i0, i0 + share, (Keys)(c.s.top + (size_t)i * PIECES), (Doubles)(c.s.seg + (size_t)i * PIECES));
  if (tid == 0) atomicMax(&st.best, best);
  if (mode == PLAIN) return;
  for (int b = tid; b < BINS; b += NT) {
    if (masses && s.mass[b]) atomicAdd(&c.s.mass[(size_t)i * BINS + b], s.mass[b]);
    if (counts && s.count[b]) atomicAdd(&c.s.count[(size_t)i * BINS + b], s.count[b]);
  }
}

// What a row's filters cut, from its histogram in LDS.  The lowest bin that can hold a kept token (of S1, where top_k and
// top_p work together), and how many tokens there are from it on: at most e^(1/32) for each unit of e^(x / 16).
template <int NT, class T> INLINE void decide(const View<T>& v, const Wants& w, bool masses, unsigned best, RowState& o) {
  auto& s = lds<NT>();
  const int tid = threadIdx.x;
  o.k = w.k;
  o.total = 0;
  // a token is kept by min_p where its logit is no lower than this
  o.floor_l = w.by_m ? (double)value_of(best) + log(w.mp) * (16.0 / v.scale) : -INFINITY;
  if (masses) {
    double x = 0;
    for (int b = tid; b < BINS; b += NT) x += (double)s.mass[b] * (s.edge[b] * (1 / UNIT));
    o.total = sum_all<NT>(x);
  }
  int t = -1, bm = -1;
  o.target = 0;
  o.above = 0;
  if (w.by_k) {
    o.target = (double)o.k;
    t = cross<NT>(o.target, 0.0, o.above);
    if (t < 0) o.k = 0;                  // fewer tokens (of any weight) than top_k
  }
  if (!o.k && w.by_p) {
    o.target = w.p * o.total;
    t = cross<NT>(o.target, -1.0, o.above);
  }
  o.by_k = o.k && t >= 0;
  o.by_p = !o.k && t >= 0;
  if (w.by_m && !(o.k && w.by_p)) {
    const unsigned f = ~(unsigned)(last_of(o.floor_l, best) >> 32);      // the key of the lowest kept logit
    const Place p = v.place(value_of(f));
    if (in_bins(p)) bm = p.bin;
  }
  o.by_m = bm >= 0 && bm >= t;
  if (bm > t) {
    t = bm;
    o.by_k = o.by_p = 0;
  }
  double from = 0;
  for (int b = tid; b < BINS; b += NT)
    if (b >= t) from += w.by_k ? (double)s.count[b] : (double)s.mass[b] * (1.0321 / UNIT);
  from = sum_all<NT>(from);
  o.mode = from <= (o.k && w.by_p ? LISTED : FEW) ? ALL : o.k && w.by_p ? DONE : CUT;      // (DONE: not by a list)
  o.bin = o.mode == ALL ? max(t, 0) : t;
}

template <class T> __global__ __launch_bounds__(DECIDE_NT) void sample_decide(Call c) {
  constexpr int NT = DECIDE_NT;
  auto& s = lds<NT>();
  const int tid = threadIdx.x, i = blockIdx.x, r = c.row0 + i;
  RowState o = c.s.row[i];
  if (o.mode == ONE) {
    if (tid == 0) {
      const bool nan = o.first == ~0ull, none = (unsigned)(o.first >> 32) == KEY_LOWEST;
      write(c.a, r, nan || none ? -1 : (int)~(unsigned)o.first, nan ? NAN : none ? -INFINITY : 0.f);
      c.s.row[i].mode = DONE;
    }
    return;
  }
  const float best = value_of(o.best);
  const View<T> v = view_of<T>(c.a, r, o.m0, o.scale);
  if (o.best == 0xffffffffu || best == -INFINITY) {      // a NaN, or no token at all
    if (tid == 0) {
      write(c.a, r, -1, best == -INFINITY ? -INFINITY : NAN);
      c.s.row[i].mode = DONE;
    }
    return;
  }
  if (v.place(best).bin >= BINS) {      // (an infinite one, too)
    if (tid == 0) {
      leave_whole(c.s, i);
      c.s.row[i].mode = DONE;
    }
    return;
  }
  if (o.mode == PLAIN) return;
  const Wants w = wants(c.a, r);
  const bool masses = w.by_p || (w.by_m && !w.by_k);
  for (int b = tid; b < BINS; b += NT) {
    s.mass[b] = c.s.mass[(size_t)i * BINS + b];
    s.count[b] = c.s.count[(size_t)i * BINS + b];
  }
  load_edges<NT>(c);
  __syncthreads();
  decide<NT>(v, w, masses, o.best, o);
  if (tid) return;
  c.s.row[i] = o;
  if (o.mode == DONE) leave_whole(c.s, i);
}

template <class T> __global__ __launch_bounds__(PART_NT) void sample_collect(Call c) {
  constexpr int NT = PART_NT;
  __shared__ unsigned long long list[PART_LIST];
  __shared__ int n, to0;
  const int tid = threadIdx.x, i = blockIdx.y;
  RowState& st = c.s.row[i];
  const int mode = st.mode, share = c.part / (NT / 64), i0 = blockIdx.x * c.part + wave_id() * share, b = st.bin;
  if (mode != ALL && mode != CUT) return;
  const View<T> v = view_of<T>(c.a, c.row0 + i, st.m0, st.scale);
  if (tid == 0) n = 0;
  if (mode == CUT) load_edges<NT>(c);
  __syncthreads();
  const Units out = (Units)(c.s.e + (size_t)i * LISTED);
  auto put = [&](unsigned long long e) __attribute__((always_inline)) {
    const int at = atomicAdd(&n, 1);
    if (at < PART_LIST) {
      list[at] = e;
    } else {
      const int to = atomicAdd(&st.n, 1);
      if (to < LISTED) out[to] = e;
    }
  };
  const Doubles seg = (Doubles)(c.s.seg + (size_t)i * PIECES);
  const Keys tops = (Keys)(c.s.top + (size_t)i * PIECES);
  if (mode == ALL) collect<true, NT>(v, b, i0, i0 + share, tops, seg, put);
  else collect<false, NT>(v, b, i0, i0 + share, tops, seg, put);
  __syncthreads();
  const int m = min(n, PART_LIST);
  if (tid == 0 && m) to0 = atomicAdd(&st.n, m);
  __syncthreads();
  for (int j = tid; j < m; j += NT)
    if (to0 + j < LISTED) out[to0 + j] = list[j];
}

template <class T> __global__ __launch_bounds__(DECIDE_NT) void sample_finish(Call c) {
  constexpr int NT = DECIDE_NT;
  auto& s = lds<NT>();
  const int tid = threadIdx.x, i = blockIdx.x, r = c.row0 + i;
  const RowState o = c.s.row[i];
  if (o.mode == DONE) return;
  if (o.n > LISTED) {
    if (tid == 0) leave_whole(c.s, i);
    return;
  }
  const Wants w = wants(c.a, r);
  const View<T> v = view_of<T>(c.a, r, o.m0, o.scale);
  load_edges<NT>(c);
  const List q{(Units)(c.s.e + (size_t)i * LISTED), (Units)(c.s.w + (size_t)i * LISTED), o.n};
  const int pieces = (v.V + PIECE - 1) / PIECE;
  if (o.mode != ALL && tid < pieces) s.seg[tid] = c.s.seg[(size_t)i * PIECES + tid];
  __syncthreads();
  if (o.mode == ALL) {
    finish_list<NT>(c.a, v, q, o.k, o.by_p || (o.k && w.by_p), w.p, o.floor_l, o.total, o.best, o.bin, w.u, r);
    return;
  }
  Cut cut = everything();
  if (o.mode == CUT && o.bin >= 0) {
    const double unit = list_weights<NT>(v, q, s.edge[o.bin] * 1.04);      // (no token of the bin weighs more: e^(1/32))
    unsigned long long last = ~0ull;
    if (o.by_k | o.by_p) last = cut_in_list<NT>(q, key_of(v.below(o.bin)), key_of(v.above(o.bin)), o.above, o.target, o.by_k, unit);
    if (o.by_m) last = min(last, last_of(o.floor_l, o.best));
    // the kept ones of the list to their pieces, in whole units
    if (tid < pieces) s.mass[tid] = 0;
    __syncthreads();
    each_of<NT>(q, [&](unsigned long long e, unsigned long long w, int) {
      if (e <= last) atomicAdd(&s.mass[(unsigned)e / PIECE], w);
    });
    __syncthreads();
    if (tid < pieces) s.seg[tid] += (double)s.mass[tid] * unit;
    __syncthreads();
    cut = Cut{~(unsigned)(last >> 32), (int)min((unsigned)last, 0x7fffffffu)};
  }
  draw<NT>(c.a, v, cut, pieces, PIECE, w.u, r);
}

// A row by one workgroup, about its maximum.
template <class T> INLINE void whole(const Call& c, int at) {
  constexpr int NT = ROW_NT, NW = NT / 64;
  auto& s = lds<NT>();
  const int tid = threadIdx.x, i = c.s.whole[1 + at], r = c.row0 + i;
  RowState o = c.s.row[i];
  const Wants w = wants(c.a, r);
  const bool inf = value_of(o.best) == INFINITY;         // infinite logits share the whole weight
  if (inf) o.best = key_of(0.f);
  View<T> v = view_of<T>(c.a, r, (double)value_of(o.best), o.scale);
  v.inf = inf;
  v.share = ((v.V + NW - 1) / NW + 255) / 256 * 256;
  load_edges<NT>(c);
  Cut cut = everything();
  const bool masses = w.by_p || (w.by_m && !w.by_k);
  double total = 0;
#pragma unroll 1
  for (int by = 0; by < 2; ++by) {       // top_k, then top_p, of the weight of S1
    if (by == 0 ? !(w.by_k || masses) : !w.by_p) continue;
    __syncthreads();
    for (int b = tid; b < BINS; b += NT) s.mass[b] = s.count[b] = 0;
    __syncthreads();
    survey<NT>(v, by || masses, !by && w.by_k, wave_id() * v.share, (wave_id() + 1) * v.share, nullptr, nullptr);
    __syncthreads();
    if (by == 0) {
      decide<NT>(v, w, masses, o.best, o);
      total = o.total;
      if (!o.k) continue;
    }
    const double target = by ? w.p * total : (double)o.k;
    double above;
    const int b = cross<NT>(target, by ? -1.0 : 0.0, above);
    if (b >= 0) cut = cut_in_row<NT>(v, b, above, target, !by);
    if (by == 0 && w.by_p) {
      sum_parts<NT>(v, cut, 0, v.V, v.share);
      total = wave_sum64(lane_id() < NW ? s.seg[lane_id()] : 0.0);
    }
  }
  if (w.by_m) {
    const unsigned f = ~(unsigned)(last_of(o.floor_l, o.best) >> 32);
    if (f > cut.key) cut = Cut{f, INT_MAX};
  }
  sum_parts<NT>(v, cut, 0, v.V, v.share);
  draw<NT>(c.a, v, cut, NW, v.share, w.u, r);
}

template <class T> __global__ __launch_bounds__(ROW_NT) void sample_whole(Call c) {
#pragma unroll 1
  for (int at = blockIdx.x; at < c.s.whole[0]; at += gridDim.x) {
    __syncthreads();
    whole<T>(c, at);
  }
}

// A call of more rows is split: what a row takes of the workspace is 0.3 MB.
constexpr int GROUP = 1024;

size_t carve(Space& s, char* p, long rows) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = p + at;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  s.whole = (int*)take((1 + rows) * 4);
  s.row = (RowState*)take(rows * sizeof(RowState));
  s.mass = (unsigned long long*)take(rows * BINS * 8);
  s.count = (unsigned*)take(rows * BINS * 4);
  s.seg = (double*)take(rows * PIECES * 8);
  s.top = (unsigned*)take(rows * PIECES * 4);
  s.edge = (double*)take(BINS * 8);
  s.e = (unsigned long long*)take((size_t)rows * LISTED * 8);
  s.w = (unsigned long long*)take((size_t)rows * LISTED * 8);
  return at;
}

template <class T> void launch_t(const SampleArgs& a, void* workspace, hipStream_t st) {
  const int group = std::min(a.rows, GROUP);
  Call c;
  c.a = a;
  carve(c.s, (char*)workspace, group);
  for (long row0 = 0; row0 < a.rows; row0 += group) {
    const int rows = (int)std::min<long>(group, a.rows - row0);
    c.row0 = (int)row0;
    // a part is no shorter than 4096 tokens (a wave of it a piece), and there are about as many as the GPU holds at once or
    // twice as many: 6 of survey's workgroups on a CU (2048 rows: 628 us with 4096 parts a group, 652 with 2048, 537 with 3072)
    const long parts = std::max(1l, std::min(3072l / rows, (a.vocab + 4095l) / 4096));
    c.part = (int)((a.vocab + parts - 1) / parts + 4095) / 4096 * 4096;
    c.parts = (a.vocab + c.part - 1) / c.part;
    const dim3 grid((unsigned)c.parts, (unsigned)rows);
    sample_begin<T><<<rows + BINS / PART_NT, PART_NT, 0, st>>>(c, rows);
    sample_survey<T><<<grid, PART_NT, 0, st>>>(c);
    sample_decide<T><<<rows, DECIDE_NT, 0, st>>>(c);
    sample_collect<T><<<grid, PART_NT, 0, st>>>(c);
    sample_finish<T><<<rows, DECIDE_NT, 0, st>>>(c);
    sample_whole<T><<<std::min(rows, 256), ROW_NT, 0, st>>>(c);
  }
}

}  // namespace

size_t sample_ws_bytes(int rows) {
  Space s;
  return carve(s, nullptr, std::min(rows, GROUP));
}

void launch_sample(int dtype, const SampleArgs& a, void* workspace, hipStream_t st) {
  if (dtype == 0) launch_t<bf16>(a, workspace, st);
  else if (dtype == 1) launch_t<float>(a, workspace, st);
  else launch_t<f16>(a, workspace, st);
}
