// Losses over sequences of token log-probabilities: paired preferences and the clipped policy loss, with their
// gradients.  float64 throughout (the losses of two query blocks are subtracted, and their difference is small), every
// sum in a fixed order.
#include "zo_internal.h"

namespace {

struct Span {
  int lo, hi;
};
// Starts that break their rule are clamped: into the rows, and up to the largest start before them.  A sequence of a large batch
// sees its own two starts and the first: in a broken batch it may take rows that are another's, never ones outside all sequences,
// and at least one sequence sees the break.  Its mark in the workspace makes the last launch, which sums what the sequences
// left there, do its block again, one sequence after another (a sequence that is not marked costs nothing more).
__device__ __forceinline__ int clamped(int start, int rows) { return min(max(start, 0), rows); }
__device__ __forceinline__ Span span_of(const int* start, int s, int rows, bool* broken, int* bad_flag) {
  const int a = start[s], b = start[s + 1];
  Span r;
  r.lo = max(clamped(a, rows), clamped(start[0], rows));
  r.hi = max(clamped(b, rows), r.lo);
  *broken = r.lo != a || r.hi != b;
  if (bad_flag && *broken) *bad_flag = 1;
  return r;
}
// Takes the sequences in order: the next one's rows.
struct InOrder {
  const int* start;
  int rows, hi;
  __device__ __forceinline__ InOrder(const int* start, int rows) : start(start), rows(rows), hi(clamped(start[0], rows)) {}
  __device__ __forceinline__ Span next(int s) {
    const int lo = hi;
    hi = max(hi, clamped(start[s + 1], rows));
    return {lo, hi};
  }
};

// A wave's sum in every lane: rows of 16 lanes by shifts, then rows onto the next ones, all in the vector unit (a shuffle goes
// through LDS, whose pipe the sums of short sequences would fill).
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V plus_moved(V v) {
  if constexpr (sizeof(V) == 4) {
    return v + __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
  } else {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    i32x2 w = __builtin_bit_cast(i32x2, v);
    w.x = __builtin_amdgcn_update_dpp(0, w.x, CTRL, ROWS, 0xf, false);
    w.y = __builtin_amdgcn_update_dpp(0, w.y, CTRL, ROWS, 0xf, false);
    return v + __builtin_bit_cast(V, w);
  }
}
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
  v = plus_moved<0x111, 0xf>(v);  // from 1, 2, 4 and 8 lanes before, within 16
  v = plus_moved<0x112, 0xf>(v);
  v = plus_moved<0x114, 0xf>(v);
  v = plus_moved<0x118, 0xf>(v);
  v = plus_moved<0x142, 0xa>(v);  // lane 15 to the second 16, 47 to the fourth
  v = plus_moved<0x143, 0xc>(v);  // lane 31 to the last 32
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
  } else {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    i32x2 w = __builtin_bit_cast(i32x2, v);
    w.x = __builtin_amdgcn_readlane(w.x, 63);
    w.y = __builtin_amdgcn_readlane(w.y, 63);
    return __builtin_bit_cast(V, w);
  }
}

// Sums over NT threads (a wave, or the workgroup), the same in every thread.  Of the N values the last M are a wave's sums
// already.
template <int NT, int N, int M = 0, typename V>
__device__ __forceinline__ void group_sum(V* v) {
#pragma unroll
  for (int k = 0; k < N - M; ++k) v[k] = wave_sum(v[k]);
  if constexpr (NT > 64) {
    __shared__ V red[N][NT / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) red[k][threadIdx.x >> 6] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = red[k][0];
#pragma unroll
      for (int j = 1; j < NT / 64; ++j) v[k] += red[k][j];
    }
  }
}

// Rows lo .. hi - 1 dealt to NT threads, U at a time so that their loads are on their way together: f(row) loads, g(row,
// whether it is one of them, what f gave) uses it.  All lanes of a wave stay in the loop, so a ballot in g counts the wave's.
template <int NT, int U = 4, typename F, typename G>
__device__ __forceinline__ void each_row(Span sp, F f, G g) {
  const int lane = threadIdx.x & 63, hi = __builtin_amdgcn_readfirstlane(sp.hi);
  for (int t0 = __builtin_amdgcn_readfirstlane(sp.lo + (int)(threadIdx.x & (NT - 64))); t0 < hi; t0 += U * NT) {
    decltype(f(0)) v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = f(min(t0 + lane + u * NT, hi - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) g(t0 + lane + u * NT, t0 + lane + u * NT < hi, v[u]);
  }
}
__device__ __forceinline__ int lanes(bool on) { return __popcll(__ballot(on)); }

// ---------------------------------------------------------------- preferences
struct PrefArgs {
  int rows, pairs, kind, average;
  double beta, margin, smoothing, weight;
  const float *logp, *ref;
  const int *labels, *start;
  double* part;  // nblk x pairs
  double* loss;
  float *rewards, *dlogp;
  int* bad_flag;
};

// The pair's loss and its slope in z.
__device__ __forceinline__ double pair_loss(const PrefArgs& a, double z, double* slope) {
  const double h = a.beta * z;
  if (a.kind == ZO_PREF_HINGE) {
    *slope = h < 1.0 ? -a.beta : h >= 1.0 ? 0.0 : h;  // NaN stays NaN
    return h < 1.0 ? 1.0 - h : h >= 1.0 ? 0.0 : h;
  }
  if (a.kind == ZO_PREF_IPO) {
    const double e = z - 0.5 / a.beta;
    *slope = 2.0 * e;
    return e * e;
  }
  // -log sigma(h) = log1p(exp(-|h|)) + max(-h, 0)
  const double u = exp(-fabs(h)), l = log1p(u);
  const double right = (h >= 0.0 ? 1.0 : u) / (1.0 + u), wrong = (h >= 0.0 ? u : 1.0) / (1.0 + u);  // sigma(h), sigma(-h)
  *slope = a.beta * (a.smoothing * right - (1.0 - a.smoothing) * wrong);
  const double keep = a.smoothing == 0.0 ? 0.0 : a.smoothing * (l + (h > 0.0 ? h : 0.0));
  return (1.0 - a.smoothing) * (l + (h < 0.0 ? -h : 0.0)) + keep;
}

// The loss of pair p of block b, sequences sp, by NT threads, its rewards and its rows' gradient.
template <int NT>
__device__ __forceinline__ double one_pair(const PrefArgs& a, int p, int b, const Span* sp) {
  const float* logp = a.logp + (size_t)b * a.rows;
  const bool first = (threadIdx.x & (NT - 1)) == 0;
  struct Row {
    float p, q;
    int y;
  };
  // Both sequences' rows together, two of each at a time.
  double v[2] = {0.0, 0.0};
  long long counts[1] = {0};  // of the chosen one, and of the other above
  const int n0 = sp[0].hi - sp[0].lo, n1 = sp[1].hi - sp[1].lo;
  for (int i = threadIdx.x & (NT - 1); i < max(n0, n1); i += 2 * NT) {
    Row r[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = min(sp[k].lo + i + u * NT, max(sp[k].hi - 1, 0));
        r[k][u] = {logp[t], a.ref ? a.ref[t] : 0.f, a.labels ? a.labels[t] : 0};
      }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (sp[k].lo + i + u * NT >= sp[k].hi || r[k][u].y < 0) continue;
        v[k] += (double)r[k][u].p - (double)r[k][u].q;
        counts[0] += 1LL << (32 * k);
      }
  }
  group_sum<NT, 2>(v);
  group_sum<NT, 1>(counts);
  const double c0 = (double)(int)counts[0], c1 = (double)(int)(counts[0] >> 32);
  const double w0 = a.average && c0 > 0.0 ? 1.0 / c0 : 1.0, w1 = a.average && c1 > 0.0 ? 1.0 / c1 : 1.0;
  const double r0 = v[0] * w0, r1 = v[1] * w1;
  double slope = 0.0, l = 0.0;
  if (c0 > 0.0 && c1 > 0.0) l = pair_loss(a, r0 - r1 - a.margin, &slope);
  if (first && a.rewards) {
    a.rewards[((size_t)b * a.pairs + p) * 2] = (float)(a.beta * r0);
    a.rewards[((size_t)b * a.pairs + p) * 2 + 1] = (float)(a.beta * r1);
  }
  if (a.dlogp) {
    slope *= a.weight / a.pairs;
    float* d = a.dlogp + (size_t)b * a.rows;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float up = (float)(k == 0 ? slope * w0 : -slope * w1);
      each_row<NT>(sp[k], [&](int t) { return a.labels ? a.labels[t] : 0; },
                   [&](int t, bool in, int y) {
                     if (in) d[t] = y >= 0 ? up : 0.f;
                   });
    }
  }
  return l;
}

// NT threads per pair and block: starts, rows, sums, the loss and the gradient one after another; 64 pairs of 2 x 256 rows 5.6 us.
template <int NT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_preference(PrefArgs a) {
  const int p = NT < 256 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, b = blockIdx.y;
  if (p >= a.pairs) return;
  const bool first = (threadIdx.x & (NT - 1)) == 0;
  Span sp[2];
  bool broken[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) sp[k] = span_of(a.start, 2 * p + k, a.rows, broken + k, first ? a.bad_flag : nullptr);
  const double l = one_pair<NT>(a, p, b, sp);
  if (first) a.part[(size_t)b * a.pairs + p] = broken[0] || broken[1] ? __builtin_nan("") : l;  // the mark
}

__global__ __launch_bounds__(256) void k_preference_total(PrefArgs a) {
  double v[1] = {0.0};
  each_row<256>(Span{0, a.pairs}, [&](int i) { return a.part[(size_t)blockIdx.x * a.pairs + i]; },
                [&](int, bool in, double l) { v[0] += in ? l : 0.0; });
  group_sum<256, 1>(v);
  if (v[0] != v[0]) {  // by a mark, or by the inputs
    int broken = 0;
    for (int s = threadIdx.x; s <= 2 * a.pairs; s += 256)
      broken |= clamped(a.start[s], a.rows) != a.start[s] || (s > 0 && a.start[s - 1] > a.start[s]);
    if (__syncthreads_or(broken)) {
      InOrder seqs(a.start, a.rows);
      v[0] = 0.0;
      for (int p = 0; p < a.pairs; ++p) {
        const Span sp[2] = {seqs.next(2 * p), seqs.next(2 * p + 1)};
        v[0] += one_pair<256>(a, p, blockIdx.x, sp);
      }
    }
  }
  if (threadIdx.x == 0) a.loss[blockIdx.x] = a.weight / a.pairs * v[0];
}

// All pairs of a block by one workgroup, a wave per pair: few rows need no second launch.
__global__ __launch_bounds__(1024) void k_preference_few(PrefArgs a) {
  __shared__ double each[16];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // Lane s has the clamped start of sequence s: at most 33.
  const int given = a.start[min(lane, 2 * a.pairs)];
  int start = clamped(given, a.rows);
  const int before = __shfl_up(start, 1, 64);
  if (__ballot(start != given || (lane > 0 && before > start))) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) start = max(start, __shfl_up(start, off, 64));  // a lane without one takes its own
    if (a.bad_flag && threadIdx.x == 0) *a.bad_flag = 1;
  }
  double l = 0.0;
  for (int p = w; p < a.pairs; p += 16) {
    const int s[3] = {__builtin_amdgcn_readlane(start, 2 * p), __builtin_amdgcn_readlane(start, 2 * p + 1),
                      __builtin_amdgcn_readlane(start, 2 * p + 2)};
    const Span sp[2] = {{s[0], s[1]}, {s[1], s[2]}};
    l += one_pair<64>(a, p, blockIdx.x, sp);
  }
  if ((threadIdx.x & 63) == 0) each[w] = l;
  __syncthreads();
  if (threadIdx.x != 0) return;
  double total = each[0];
#pragma unroll
  for (int j = 1; j < 16; ++j) total += each[j];
  a.loss[blockIdx.x] = a.weight / a.pairs * total;
}

// ---------------------------------------------------------------- policy
struct PolicyArgs {
  int nblk, rows, nseq, aggregate, per_token;
  double low, high, kl, weight;
  const float *logp, *old, *ref, *adv;
  const int *labels, *start;
  int ncount;
  int* counted;   // rows that count, in ncount parts (token, with a gradient)
  int* of_seq;    // and of each sequence
  double* part;   // nblk x nseq x 3
  double *loss, *stats;
  float* dlogp;
  int* bad_flag;
};

struct PolicyRow {
  float old, ref, adv;
  int y;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, int t, int s) {
  return {a.old[t], a.ref ? a.ref[t] : 0.f, a.adv[a.per_token ? t : s], a.labels ? a.labels[t] : 0};
}

// exp(d) = 2^n (1 + r + q): d = n log 2 + r with |r| <= log(2) / 2, and q = exp(r) - r - 1 by its series, r^2 (1/2! + r/3! + ... +
// r^11/13!), 2^-52 of it left out.  Below -800 exp is 0.  n stops at 1023, where r grows instead and 2^n (1 + r + q) beyond all numbers
// with it; infinity and NaN stay in r.
struct Exponential {
  double r, q;
  int n;
  __device__ __forceinline__ explicit Exponential(double d) {
    constexpr double over[12] = {1.0 / 6227020800.0, 1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0,
                                 1.0 / 5040.0,       1.0 / 720.0,       1.0 / 120.0,      1.0 / 24.0,      1.0 / 6.0,      0.5};
    const double x = d < -800.0 ? -800.0 : d;
    const double e = fmin(rint(x * 1.4426950408889634), 1023.0);
    r = fma(-e, 2.3190468138462996e-17, fma(-e, 0.6931471805599453, x));  // log 2 in two parts
    double p = over[0];
#pragma unroll
    for (int i = 1; i < 12; ++i) p = fma(p, r, over[i]);
    q = r * r * p;
    n = (int)e;
  }
  __device__ __forceinline__ double value() const { return ldexp(1.0 + (r + q), n); }
};

// k = exp(d) - d - 1 and m = exp(d) - 1, without the differences that would cancel where the models nearly agree (at d = 1e-6 k would
// keep four digits): with t = 2^n, k = t q + (t - 1 + (t r - d)), which is q at n = 0; elsewhere k is at least 0.047 exp(d).
__device__ __forceinline__ double kl_term(double d, double* m) {
  const Exponential e(d);
  const double t = ldexp(1.0, e.n), t1 = t - 1.0;
  *m = fma(t, e.r + e.q, t1);
  return fma(t, e.q, t1 + fma(t, e.r, -fmin(d, 1e300)));  // at d = infinity r alone is infinite
}

// Adds a row that counts to (loss, k), says whether it is clipped and returns its slope.
template <bool GRAD>
__device__ __forceinline__ double policy_term(const PolicyArgs& a, float logp, const PolicyRow& x, double* v, bool* clipped) {
  const double p = logp, A = x.adv, r = Exponential(p - (double)x.old).value();
  const double c = fmin(fmax(r, 1.0 - a.low), 1.0 + a.high);
  const double plain = r * A, kept = c * A;  // where r is NaN, plain is
  const bool cut = plain > kept;
  double gain = cut ? kept : plain, rise = 0.0;
  if constexpr (GRAD) rise = cut ? 0.0 : plain;
  if (a.ref) {
    double m;
    const double k = kl_term((double)x.ref - p, &m);
    if (a.kl != 0.0) {  // else an infinite k is only reported
      gain -= a.kl * k;
      if constexpr (GRAD) rise += a.kl * m;
    }
    v[1] += k;
  }
  v[0] -= gain;
  *clipped = cut;
  return -rise;
}

__device__ __forceinline__ double inverse(double n) { return n > 0.0 ? 1.0 / n : 0.0; }

// The rows that count among all: sequences follow one another, so they are rows start[0] .. start[nseq] - 1.
__global__ __launch_bounds__(256) void k_policy_count(PolicyArgs a) {
  const int lo = min(max(a.start[0], 0), a.rows), hi = min(max(a.start[a.nseq], lo), a.rows);
  const int each = (hi - lo + a.ncount - 1) / a.ncount;
  Span sp = {min(lo + (int)blockIdx.x * each, hi), 0};
  sp.hi = min(sp.lo + each, hi);
  int n[1] = {0};
  each_row<256>(sp, [&](int t) { return a.labels ? a.labels[t] : 0; }, [&](int, bool in, int y) { n[0] += lanes(in && y >= 0); });
  group_sum<256, 1, 1>(n);
  if (threadIdx.x == 0) a.counted[blockIdx.x] = n[0];
}

// NT threads take a sequence, under NB blocks at once: what the blocks share is loaded once.  Float64 bounds it beside its start:
// 112 vector instructions a row and block, two exponentials and k about half of them.  512 sequences of up to 1024 rows under 16
// blocks, a call in a graph: 21.3 us (with one block a workgroup 24.0, four 21.8), twice the rows 12.6 more.
template <int NT, int NB, bool GRAD>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_policy(PolicyArgs a) {
  const int s = NT < 256 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, b0 = blockIdx.y * NB;
  double n[1] = {0.0};
  if (GRAD && a.aggregate == ZO_AGG_TOKEN) {
    for (int i = threadIdx.x & (NT - 1); i < a.ncount; i += NT) n[0] += a.counted[i];
    group_sum<NT, 1>(n);
  }
  if (s >= a.nseq) return;
  const bool first = (threadIdx.x & (NT - 1)) == 0;
  bool broken;
  const Span sp = span_of(a.start, s, a.rows, &broken, first && b0 == 0 ? a.bad_flag : nullptr);
  if (GRAD && a.aggregate == ZO_AGG_SEQUENCE) {
    int c[1] = {0};
    each_row<NT>(sp, [&](int t) { return a.labels ? a.labels[t] : 0; }, [&](int, bool in, int y) { c[0] += lanes(in && y >= 0); });
    group_sum<NT, 1, 1>(c);
    n[0] = (double)c[0] * a.nseq;
  }
  const double share = a.weight * (a.aggregate == ZO_AGG_SUM ? 1.0 : inverse(n[0]));  // of the gradient
  double v[3 * NB + 1];  // (loss, k) of each block; how many are clipped in each; how many count
#pragma unroll
  for (int k = 0; k < 2 * NB; ++k) v[k] = 0.0;
  int clipped[NB] = {}, count = 0;
  struct Row {
    PolicyRow x;
    float p[NB];
  };
  each_row<NT, 1>(
      sp,
      [&](int t) {
        Row r = {policy_row(a, t, s), {}};
#pragma unroll
        for (int k = 0; k < NB; ++k) r.p[k] = a.logp[(size_t)min(b0 + k, a.nblk - 1) * a.rows + t];
        return r;
      },
      [&](int t, bool in, const Row& r) {
        const bool on = in && r.x.y >= 0;
        bool cut[NB] = {};
        count += lanes(on);
        double slope[NB] = {};
        if (on)
#pragma unroll
          for (int k = 0; k < NB; ++k) slope[k] = policy_term<GRAD>(a, r.p[k], r.x, v + 2 * k, cut + k);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          clipped[k] += lanes(cut[k]);
          if (GRAD && in && b0 + k < a.nblk) a.dlogp[(size_t)(b0 + k) * a.rows + t] = on ? (float)(slope[k] * share) : 0.f;
        }
      });
#pragma unroll
  for (int k = 0; k < NB; ++k) v[2 * NB + k] = clipped[k];
  v[3 * NB] = count;
  group_sum<NT, 3 * NB + 1, NB + 1>(v);
  if (!first) return;
  if (b0 == 0) a.of_seq[s] = broken ? -1 : (int)v[3 * NB];  // the mark
  const double mine = a.aggregate == ZO_AGG_SEQUENCE ? inverse(v[3 * NB] * a.nseq) : 1.0;
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    if (b0 + k >= a.nblk) break;
    double* to = a.part + ((size_t)(b0 + k) * a.nseq + s) * 3;
    to[0] = v[2 * k] * mine;
    to[1] = v[2 * k + 1];
    to[2] = v[2 * NB + k];
  }
}

// All sequences of a block whose starts are broken, one after another by 256 threads: v gets the sums of the loss, of k and of
// the clipped rows, and the rows that count.
__device__ __forceinline__ void in_order(const PolicyArgs& a, double* v) {
  auto label = [&](int t) { return a.labels ? a.labels[t] : 0; };
  int n[1] = {0};
  InOrder all(a.start, a.rows);
  for (int s = 0; s < a.nseq; ++s) each_row<256>(all.next(s), label, [&](int, bool in, int y) { n[0] += lanes(in && y >= 0); });
  group_sum<256, 1, 1>(n);
  v[0] = v[1] = v[2] = 0.0;
  v[3] = n[0];
  const size_t block = (size_t)blockIdx.x * a.rows;
  InOrder seqs(a.start, a.rows);
  for (int s = 0; s < a.nseq; ++s) {
    const Span sp = seqs.next(s);
    double share = a.aggregate == ZO_AGG_TOKEN ? inverse(v[3]) : 1.0;
    if (a.aggregate == ZO_AGG_SEQUENCE) {
      int c[1] = {0};
      each_row<256>(sp, label, [&](int, bool in, int y) { c[0] += lanes(in && y >= 0); });
      group_sum<256, 1, 1>(c);
      share = inverse((double)c[0] * a.nseq);
    }
    for (int t = sp.lo + (int)threadIdx.x; t < sp.hi; t += 256) {
      double one[2] = {0.0, 0.0}, slope = 0.0;
      bool cut = false;
      const PolicyRow x = policy_row(a, t, s);
      if (x.y >= 0) slope = policy_term<true>(a, a.logp[block + t], x, one, &cut);
      v[0] += a.aggregate == ZO_AGG_SEQUENCE ? one[0] * share : one[0];
      v[1] += one[1];
      v[2] += cut ? 1.0 : 0.0;
      if (a.dlogp) a.dlogp[block + t] = (float)(slope * share * a.weight);
    }
  }
  group_sum<256, 3>(v);
}

__global__ __launch_bounds__(256) void k_policy_total(PolicyArgs a) {
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  const double* part = a.part + (size_t)blockIdx.x * a.nseq * 3;
  struct Row {
    double x[3];
    int n;
  };
  each_row<256>(
      Span{0, a.nseq}, [&](int i) { return Row{{part[(size_t)i * 3], part[(size_t)i * 3 + 1], part[(size_t)i * 3 + 2]}, a.of_seq[i]}; },
      [&](int, bool in, const Row& r) {
        if (!in) return;
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] += r.x[k];
        v[3] += r.n < 0 ? __builtin_nan("") : (double)r.n;
      });
  group_sum<256, 4>(v);
  if (v[3] != v[3]) in_order(a, v);
  if (threadIdx.x != 0) return;
  a.loss[blockIdx.x] = a.weight * (a.aggregate == ZO_AGG_TOKEN ? v[0] * inverse(v[3]) : v[0]);
  if (a.stats) {
    a.stats[2 * blockIdx.x] = v[1] * inverse(v[3]);
    a.stats[2 * blockIdx.x + 1] = v[2] * inverse(v[3]);
  }
}

// All rows of a block by one workgroup, a thread per row: few rows need no other launch (1600 rows 5.0 us).  A row's sequence is
// the last one that starts at it or before.
constexpr int FEW_SEQS = 256, FEW_ROWS = 4;  // sequences, and rows of a thread
__global__ __launch_bounds__(1024) void k_policy_few(PolicyArgs a) {
  constexpr int WAVES = FEW_SEQS / 64 + 1;  // that have starts
  __shared__ int start[FEW_SEQS + 1], count[FEW_SEQS], broken[WAVES];
  const int b = blockIdx.x, t0 = threadIdx.x;
  if (t0 < 64 * WAVES) {
    const int s = min(t0, a.nseq), given = a.start[s], before = a.start[max(s - 1, 0)];
    start[s] = clamped(given, a.rows);
    if (t0 < a.nseq) count[t0] = 0;
    const unsigned long long bad = __ballot(clamped(given, a.rows) != given || (s > 0 && before > given));
    if ((t0 & 63) == 0) broken[t0 >> 6] = bad != 0;
  }
  __syncthreads();
  const int lo = start[0];
  int hi = start[a.nseq], bad = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) bad |= broken[w];
  if (bad) {
    if (t0 == 0) {
      for (int s = 1; s <= a.nseq; ++s) start[s] = max(start[s], start[s - 1]);
      if (a.bad_flag) *a.bad_flag = 1;
    }
    __syncthreads();
    hi = start[a.nseq];
  }
  const bool by_seq = a.aggregate == ZO_AGG_SEQUENCE;
  struct Row {
    PolicyRow x;
    float p;
    int s;
  } r[FEW_ROWS];
#pragma unroll
  for (int k = 0; k < FEW_ROWS; ++k) {
    if (lo + k * 1024 >= hi) break;
    const int t = min(lo + k * 1024 + t0, hi - 1);
    r[k].s = 0;
    if (by_seq || !a.per_token) {  // start[s] <= t < start[s + 1]
      int first = 0, behind = a.nseq;
      while (behind - first > 1) {
        const int m = (first + behind) >> 1;
        if (start[m] <= t) first = m;
        else behind = m;
      }
      r[k].s = first;
    }
    r[k].x = policy_row(a, t, r[k].s);
    r[k].p = a.logp[(size_t)b * a.rows + t];
    if (lo + k * 1024 + t0 >= hi) r[k].x.y = -1;
    if (by_seq && r[k].x.y >= 0) atomicAdd(&count[r[k].s], 1);  // whole numbers: in any order
  }
  int n[1] = {0}, clipped = 0;
#pragma unroll
  for (int k = 0; k < FEW_ROWS; ++k)
    if (lo + k * 1024 < hi) n[0] += lanes(r[k].x.y >= 0);
  group_sum<1024, 1, 1>(n);  // and the counts above are whole
  const double N = n[0];
  double v[3] = {0.0, 0.0, 0.0};
#pragma unroll
  for (int k = 0; k < FEW_ROWS; ++k) {
    if (lo + k * 1024 >= hi) break;
    double up = 0.0;
    bool cut = false;
    if (r[k].x.y >= 0) {
      double one[2] = {0.0, 0.0};
      const double slope = policy_term<true>(a, r[k].p, r[k].x, one, &cut);
      const double share = a.aggregate == ZO_AGG_SUM ? 1.0 : inverse(by_seq ? (double)count[r[k].s] * a.nseq : N);
      v[0] += by_seq ? one[0] * share : one[0];
      v[1] += one[1];
      up = slope * share * a.weight;
    }
    clipped += lanes(cut);
    const int t = lo + k * 1024 + t0;
    if (a.dlogp && t < hi) a.dlogp[(size_t)b * a.rows + t] = (float)up;
  }
  v[2] = clipped;
  group_sum<1024, 3, 1>(v);
  if (t0 != 0) return;
  a.loss[b] = a.weight * (a.aggregate == ZO_AGG_TOKEN ? v[0] * inverse(N) : v[0]);
  if (a.stats) {
    a.stats[2 * b] = v[1] * inverse(N);
    a.stats[2 * b + 1] = v[2] * inverse(N);
  }
}

}  // namespace

int zo_preference_loss_launch(int nblk, int rows, int pairs, int kind, int average, double beta, double margin, double smoothing,
                              double weight, const float* logp, const float* ref_logp, const int* labels, const int* seq_start,
                              double* loss, float* rewards, float* dlogp, int* bad_flag, void* ws, hipStream_t stream,
                              size_t* ws_needed) {
  // us a call with one launch and with two, from Python one after another (the host bounds them) and in a graph: 2 pairs of 200
  // rows 7.6, 11.9 and 5.1, 6.6; 8 of 256 7.7, 12.0 and 5.7, 6.6; 1 of 1024 8.5, 11.9 and 8.8, 6.6; but 32 pairs, two a wave, 10.8,
  // 11.9 and 11.2, 6.4.
  const bool few = rows <= 2048 && rows <= 1024LL * pairs && pairs <= 16;
  if (ws_needed) {
    *ws_needed = few ? 0 : zo_align256((size_t)nblk * pairs * sizeof(double));
    return ZO_OK;
  }
  const PrefArgs a = {rows, pairs, kind, average, beta, margin, smoothing, weight, logp, ref_logp, labels, seq_start, (double*)ws,
                      loss, rewards, dlogp, bad_flag};
  if (few) {
    hipLaunchKernelGGL(k_preference_few, dim3(nblk), dim3(1024), 0, stream, a);
    return zo_hip_status(hipGetLastError(), "k_preference_few");
  }
  // us with a wave, 256 and 1024 threads a pair: 8192 pairs of 2 x 250 rows 19.5, 36.6, -; 2048 of them 9.9, 13.6, -; 512 of 2 x
  // 500 12.1, 8.8, -; 128 of 2 x 1000 18.3, 8.7, 10.4; 16 of 2 x 3000 -, 15.4, 11.4.
  const long long mean = rows / (2 * pairs), groups = (long long)nblk * pairs;
  if (mean <= 64 || groups >= 8 * mean) hipLaunchKernelGGL(k_preference<64>, dim3((pairs + 3) / 4, nblk), dim3(256), 0, stream, a);
  else if (mean <= 1500) hipLaunchKernelGGL(k_preference<256>, dim3(pairs, nblk), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(k_preference<1024>, dim3(pairs, nblk), dim3(1024), 0, stream, a);
  const int st = zo_hip_status(hipGetLastError(), "k_preference");
  if (st != ZO_OK) return st;
  hipLaunchKernelGGL(k_preference_total, dim3(nblk), dim3(256), 0, stream, a);
  return zo_hip_status(hipGetLastError(), "k_preference_total");
}

int zo_policy_loss_launch(int nblk, int rows, int nseq, int aggregate, int per_token, double clip_low, double clip_high,
                          double kl_coef, double weight, const float* logp, const float* old_logp, const float* ref_logp,
                          const float* advantage, const int* labels, const int* seq_start, double* loss, double* stats,
                          float* dlogp, int* bad_flag, void* ws, hipStream_t stream, size_t* ws_needed) {
  // us a call with a KL term and gradients in one launch and in two (three for ZO_AGG_TOKEN), from Python one after another (the host
  // bounds the latter) and in a graph.  Sequence means, 16 sequences of 100 rows: 8.4, 12.3 and 6.2, 6.3; of 250: 10.3, 12.1 and 10.8,
  // 6.2.  Token means: 8.3, 14.6 and 5.7, 8.7; 8.8, 15.3 and 9.3, 9.8.  16 of 500 rows, 8 a thread, 18 in a graph.
  const bool few = rows <= 1024 * FEW_ROWS && nseq <= FEW_SEQS;
  const int ncount = rows < 256 * 4096 ? (rows + 4095) / 4096 + (rows == 0) : 256;
  WsCarver w(ws);
  int* counted = (int*)w.take((size_t)ncount * sizeof(int));
  int* of_seq = (int*)w.take((size_t)nseq * sizeof(int));
  double* part = (double*)w.take((size_t)nblk * nseq * 3 * sizeof(double));
  if (ws_needed) {
    *ws_needed = few ? 0 : w.off;
    return ZO_OK;
  }
  const PolicyArgs a = {nblk, rows, nseq, aggregate, per_token, clip_low, clip_high, kl_coef, weight, logp, old_logp, ref_logp,
                        advantage, labels, seq_start, ncount, counted, of_seq, part, loss, stats, dlogp, bad_flag};
  if (few) {
    hipLaunchKernelGGL(k_policy_few, dim3(nblk), dim3(1024), 0, stream, a);
    return zo_hip_status(hipGetLastError(), "k_policy_few");
  }
  int st = ZO_OK;
  if (dlogp && aggregate == ZO_AGG_TOKEN) {
    hipLaunchKernelGGL(k_policy_count, dim3(ncount), dim3(256), 0, stream, a);
    if ((st = zo_hip_status(hipGetLastError(), "k_policy_count")) != ZO_OK) return st;
  }
  // us in a graph with a wave, 256 and 1024 threads a sequence (and two blocks, but with 1024), with a KL term and, for one block, its
  // gradient: 4096 sequences of 200 rows 18.0, 19.4, 51.0; 1024 of 200 12.6, 11.5, 19.1; of 600 16.1, 13.1, 20.5; 1024 of 500 under 16
  // blocks 30.1, 30.8, 135; 256 of 4000 67.9, 25.2, 17.0; 256 of 600 under 16 blocks 14.2, 13.6, 37.1; 16 of 2000 26.3, 13.4, 12.0.
  const long long mean = rows / nseq;
  const int nb = nblk >= 2 ? 2 : 1, y = (nblk + nb - 1) / nb;
  auto go = [&](auto grad, auto none, dim3 grid, int threads) {
    hipLaunchKernelGGL(dlogp ? grad : none, grid, dim3(threads), 0, stream, a);
  };
  if (mean <= 128 || (mean <= 512 && (long long)nseq * y >= 16 * mean)) {
    const dim3 grid((nseq + 3) / 4, y);
    nb == 2 ? go(k_policy<64, 2, true>, k_policy<64, 2, false>, grid, 256) : go(k_policy<64, 1, true>, k_policy<64, 1, false>, grid, 256);
  } else if (mean <= 1000 || (long long)nseq * nblk > 2048) {
    const dim3 grid(nseq, y);
    nb == 2 ? go(k_policy<256, 2, true>, k_policy<256, 2, false>, grid, 256)
            : go(k_policy<256, 1, true>, k_policy<256, 1, false>, grid, 256);
  } else {
    go(k_policy<1024, 1, true>, k_policy<1024, 1, false>, dim3(nseq, nblk), 1024);
  }
  st = zo_hip_status(hipGetLastError(), "k_policy");
  if (st != ZO_OK) return st;
  hipLaunchKernelGGL(k_policy_total, dim3(nblk), dim3(256), 0, stream, a);
  return zo_hip_status(hipGetLastError(), "k_policy_total");
}
