// Losses over sequences of token log-probabilities: paired preferences and the clipped policy loss, with their
// gradients.  float64 throughout; every sum in a fixed order.
#include "zo_internal.h"

namespace {

struct Span {
  int lo, hi;
};
// A sequence's rows, clamped into the tensors.
__device__ __forceinline__ Span span_of(const int* start, int s, int rows, int* bad_flag) {
  const int a = start[s], b = start[s + 1];
  Span r;
  r.lo = min(max(a, 0), rows);
  r.hi = min(max(b, r.lo), rows);
  if (bad_flag && (r.lo != a || r.hi != b)) *bad_flag = 1;
  return r;
}

// Sums over a workgroup of 256, the same in every thread.
template <int N>
__device__ __forceinline__ void group_sum(double* v) {
  __shared__ double red[N][4];
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v[k] += __shfl_xor(v[k], off, 64);
    if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = (red[k][0] + red[k][1]) + (red[k][2] + red[k][3]);
  __syncthreads();
}

struct PrefArgs {
  int rows, pairs, kind, average;
  double beta, margin, smoothing, weight;
  const float *logp, *ref;
  const int *labels, *start;
  double* part;
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

// A workgroup per pair and block.
__global__ __launch_bounds__(256) void k_preference(PrefArgs a) {
  const int p = blockIdx.x, b = blockIdx.y;
  const float* logp = a.logp + (size_t)b * a.rows;
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  Span sp[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    sp[k] = span_of(a.start, 2 * p + k, a.rows, threadIdx.x == 0 ? a.bad_flag : nullptr);
    for (int t = sp[k].lo + threadIdx.x; t < sp[k].hi; t += 256) {
      if (a.labels && a.labels[t] < 0) continue;
      v[k] += (double)logp[t] - (a.ref ? (double)a.ref[t] : 0.0);
      v[2 + k] += 1.0;
    }
  }
  group_sum<4>(v);
  const double w0 = a.average && v[2] > 0.0 ? 1.0 / v[2] : 1.0, w1 = a.average && v[3] > 0.0 ? 1.0 / v[3] : 1.0;
  const double r0 = v[0] * w0, r1 = v[1] * w1;
  double slope = 0.0, l = 0.0;
  if (v[2] > 0.0 && v[3] > 0.0) l = pair_loss(a, r0 - r1 - a.margin, &slope);
  if (threadIdx.x == 0) {
    a.part[(size_t)b * a.pairs + p] = l;
    if (a.rewards) {
      a.rewards[((size_t)b * a.pairs + p) * 2] = (float)(a.beta * r0);
      a.rewards[((size_t)b * a.pairs + p) * 2 + 1] = (float)(a.beta * r1);
    }
  }
  if (!a.dlogp) return;
  slope *= a.weight / a.pairs;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float up = (float)(k == 0 ? slope * w0 : -slope * w1);
    for (int t = sp[k].lo + threadIdx.x; t < sp[k].hi; t += 256)
      a.dlogp[(size_t)b * a.rows + t] = !a.labels || a.labels[t] >= 0 ? up : 0.f;
  }
}

// out[b] = factor sum of part[b]: one workgroup per block.
__global__ __launch_bounds__(256) void k_preference_total(const double* part, int n, double factor, double* out) {
  double v[1] = {0.0};
  for (int i = threadIdx.x; i < n; i += 256) v[0] += part[(size_t)blockIdx.x * n + i];
  group_sum<1>(v);
  if (threadIdx.x == 0) out[blockIdx.x] = factor * v[0];
}

struct PolicyArgs {
  int rows, nseq, aggregate, per_token;
  double low, high, kl, weight;
  const float *logp, *old, *ref, *adv;
  const int *labels, *start;
  int* count;     // rows that count, per sequence
  double* part;   // nblk x nseq x 3
  float* dlogp;
  int* bad_flag;
};

__global__ __launch_bounds__(256) void k_policy_count(PolicyArgs a) {
  const Span sp = span_of(a.start, blockIdx.x, a.rows, threadIdx.x == 0 ? a.bad_flag : nullptr);
  double v[1] = {0.0};
  for (int t = sp.lo + threadIdx.x; t < sp.hi; t += 256) v[0] += !a.labels || a.labels[t] >= 0 ? 1.0 : 0.0;
  group_sum<1>(v);
  if (threadIdx.x == 0) a.count[blockIdx.x] = (int)v[0];
}

// A workgroup per sequence and block.
__global__ __launch_bounds__(256) void k_policy(PolicyArgs a) {
  const int s = blockIdx.x, b = blockIdx.y;
  double n[1] = {0.0};
  for (int i = threadIdx.x; i < a.nseq; i += 256) n[0] += a.count[i];
  group_sum<1>(n);
  const double mine = a.count[s];
  const double share = a.weight * (a.aggregate == ZO_AGG_TOKEN ? (n[0] > 0.0 ? 1.0 / n[0] : 0.0)
                                   : a.aggregate == ZO_AGG_SEQUENCE ? (mine > 0.0 ? 1.0 / mine / a.nseq : 0.0) : 1.0);
  const Span sp = span_of(a.start, s, a.rows, nullptr);
  const float* logp = a.logp + (size_t)b * a.rows;
  double v[3] = {0.0, 0.0, 0.0};
  for (int t = sp.lo + threadIdx.x; t < sp.hi; t += 256) {
    float up = 0.f;
    if (!a.labels || a.labels[t] >= 0) {
      const double p = logp[t], A = a.adv[a.per_token ? t : s];
      const double r = exp(p - (double)a.old[t]);
      const double c = r < 1.0 - a.low ? 1.0 - a.low : (r > 1.0 + a.high ? 1.0 + a.high : r);
      const double plain = r * A, kept = c * A;
      const bool cut = plain > kept;
      double l = cut ? -kept : -plain, slope = cut ? 0.0 : -plain;
      if (a.ref) {
        const double d = (double)a.ref[t] - p, e = exp(d), k = d < __builtin_inf() ? e - d - 1.0 : e;  // infinite at d = inf
        l += a.kl * k;
        slope += a.kl * (1.0 - e);
        v[1] += k;
      }
      v[0] += l;
      v[2] += cut ? 1.0 : 0.0;
      up = (float)(slope * share);
    }
    if (a.dlogp) a.dlogp[(size_t)b * a.rows + t] = up;
  }
  group_sum<3>(v);
  if (threadIdx.x == 0) {
    double* to = a.part + ((size_t)b * a.nseq + s) * 3;
    to[0] = v[0] * share;
    to[1] = n[0] > 0.0 ? v[1] / n[0] : 0.0;
    to[2] = n[0] > 0.0 ? v[2] / n[0] : 0.0;
  }
}

__global__ __launch_bounds__(256) void k_policy_total(const double* part, int n, double* loss, double* stats) {
  double v[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < n; i += 256)
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] += part[((size_t)blockIdx.x * n + i) * 3 + k];
  group_sum<3>(v);
  if (threadIdx.x == 0) {
    loss[blockIdx.x] = v[0];
    if (stats) {
      stats[2 * blockIdx.x] = v[1];
      stats[2 * blockIdx.x + 1] = v[2];
    }
  }
}

}  // namespace

int zo_preference_loss_launch(int nblk, int rows, int pairs, int kind, int average, double beta, double margin, double smoothing,
                              double weight, const float* logp, const float* ref_logp, const int* labels, const int* seq_start,
                              double* loss, float* rewards, float* dlogp, int* bad_flag, void* ws, hipStream_t stream,
                              size_t* ws_needed) {
  WsCarver w(ws);
  double* part = (double*)w.take((size_t)nblk * pairs * sizeof(double));
  if (ws_needed) {
    *ws_needed = w.off;
    return ZO_OK;
  }
  const PrefArgs a = {rows, pairs, kind, average, beta, margin, smoothing, weight, logp, ref_logp, labels, seq_start, part,
                      rewards, dlogp, bad_flag};
  hipLaunchKernelGGL(k_preference, dim3(pairs, nblk), dim3(256), 0, stream, a);
  const int st = zo_hip_status(hipGetLastError(), "k_preference");
  if (st != ZO_OK) return st;
  hipLaunchKernelGGL(k_preference_total, dim3(nblk), dim3(256), 0, stream, part, pairs, weight / pairs, loss);
  return zo_hip_status(hipGetLastError(), "k_preference_total");
}

int zo_policy_loss_launch(int nblk, int rows, int nseq, int aggregate, int per_token, double clip_low, double clip_high,
                          double kl_coef, double weight, const float* logp, const float* old_logp, const float* ref_logp,
                          const float* advantage, const int* labels, const int* seq_start, double* loss, double* stats,
                          float* dlogp, int* bad_flag, void* ws, hipStream_t stream, size_t* ws_needed) {
  WsCarver w(ws);
  int* count = (int*)w.take((size_t)nseq * sizeof(int));
  double* part = (double*)w.take((size_t)nblk * nseq * 3 * sizeof(double));
  if (ws_needed) {
    *ws_needed = w.off;
    return ZO_OK;
  }
  const PolicyArgs a = {rows, nseq, aggregate, per_token, clip_low, clip_high, kl_coef, weight, logp, old_logp, ref_logp,
                        advantage, labels, seq_start, count, part, dlogp, bad_flag};
  hipLaunchKernelGGL(k_policy_count, dim3(nseq), dim3(256), 0, stream, a);
  int st = zo_hip_status(hipGetLastError(), "k_policy_count");
  if (st != ZO_OK) return st;
  hipLaunchKernelGGL(k_policy, dim3(nseq, nblk), dim3(256), 0, stream, a);
  if ((st = zo_hip_status(hipGetLastError(), "k_policy")) != ZO_OK) return st;
  hipLaunchKernelGGL(k_policy_total, dim3(nblk), dim3(256), 0, stream, part, nseq, loss, stats);
  return zo_hip_status(hipGetLastError(), "k_policy_total");
}
