// Log-probabilities of labelled tokens over the vocabulary, and the logits' gradient.
#include "zo_internal.h"

#include <type_traits>

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LEAST = -16777216.f;  // powers of one pass stay between +-2^24, where their rounding is at most a half

template <int DT>
struct Elem {
  static constexpr int SIZE = DT == ZO_F32 ? 4 : 2;
  static constexpr int N = 16 / SIZE;  // elements of a 16-byte word

  static __device__ __forceinline__ float load(const char* p) {
    if constexpr (DT == ZO_F32) return *(const float*)p;
    else if constexpr (DT == ZO_BF16) return bf16_to_f32(*(const bf16_t*)p);
    else return f16_to_f32(*(const uint16_t*)p);
  }
  static __device__ __forceinline__ void store(char* p, float v) {
    if constexpr (DT == ZO_F32) *(float*)p = v;
    else if constexpr (DT == ZO_BF16) *(bf16_t*)p = f32_to_bf16(v);
    else *(uint16_t*)p = f32_to_f16(v);
  }
  static __device__ __forceinline__ void widen(const u32x4& w, float* x) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DT == ZO_F32) {
        x[k] = __uint_as_float(w[k]);
      } else if constexpr (DT == ZO_BF16) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
      } else {
        x[2 * k] = f16_to_f32((uint16_t)w[k]);
        x[2 * k + 1] = f16_to_f32((uint16_t)(w[k] >> 16));
      }
    }
  }
  static __device__ __forceinline__ u32x4 narrow(const float* x) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DT == ZO_F32) w[k] = __float_as_uint(x[k]);
      else if constexpr (DT == ZO_BF16) w[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
      else w[k] = pack_f16x2(x[2 * k], x[2 * k + 1]);
    }
    return w;
  }
};

// The 16-byte words of a row: elements before the first, words, elements behind the last.
struct RowWords {
  int head, words, tail;
};
template <int DT>
__device__ __forceinline__ RowWords row_words(const char* x, int vocab) {
  RowWords r;
  r.head = min((int)((16 - ((uintptr_t)x & 15)) & 15) / Elem<DT>::SIZE, vocab);
  r.words = (vocab - r.head) / Elem<DT>::N;
  r.tail = vocab - r.head - r.words * Elem<DT>::N;
  return r;
}

// Sum of exp2(c x) relative to 2^R: s = sum of 2^(c x - R).  R only grows; every term is one multiply-add (c x is exact
// in it) and one exponential.  R is a value of its own, not the rounding of a product that is formed again, so that what
// it was rounded by cancels: the row's log-sum-exp is (R + log2 s) log 2.  For that the product that becomes R may not be
// contracted into the difference that the sum is scaled by: R there would be the product before its rounding, and a carried sum
// 2^(R's rounding) off, 4 % at logits of 10^6.  R begins at -2^24 and not at the lowest value: were a
// masked logit of -1e30 some thread's own R, the rounding of its product would be a power of 2^70, its exponential infinite,
// and infinity times the 0 that raise() scales it by NaN.  As it is such a logit adds 0.
struct Sum {
  float R, s;
  __device__ __forceinline__ void raise(float to) {
#pragma clang fp contract(off)
    s *= __builtin_amdgcn_exp2f(R - to);
    R = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const float* x, float c) {
#pragma clang fp contract(off)
    float m = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, x[k]);
    m *= c;
    if (m > R) raise(m);
    float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < N; ++k) p[k & 3] += __builtin_amdgcn_exp2f(fmaf(x[k], c, -R));
    s += (p[0] + p[1]) + (p[2] + p[3]);
  }
};

// Largest value and sum over the NT threads of a row: a wave, or the workgroup.
template <int NT>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  if constexpr (NT > 64) {
    __shared__ float red[NT / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) v = fmaxf(v, red[k]);
  }
  return v;
}
template <int NT>
__device__ __forceinline__ float group_total(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if constexpr (NT > 64) {
    __shared__ float red[NT / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) v += red[k];
  }
  return v;
}

// The sum over words lo .. hi - 1 of a row, and with `edges` over its elements before and behind the words.  Whole steps of
// U NT words need no checks, so the next step's loads stay on their way while this one's are added.
template <int DT, int NT>
__device__ __forceinline__ Sum row_sum(const char* x, const RowWords& r, int vocab, int lo, int hi, bool edges, float c) {
  using EL = Elem<DT>;
  constexpr int U = 2;
  const int tid = threadIdx.x & (NT - 1), steps = (hi - lo) / (U * NT);
  const u32x4* words = (const u32x4*)(x + r.head * EL::SIZE) + lo + tid;
  const int rest = hi - lo - tid;  // words from this thread's first on
  Sum sum = {LEAST, 0.f};
  u32x4 last[U], w[U], next[U];
  float edge[2] = {-__builtin_inff(), -__builtin_inff()};
  if (edges && tid < r.head) edge[0] = EL::load(x + tid * EL::SIZE);
  if (edges && tid < r.tail) edge[1] = EL::load(x + ((size_t)vocab - 1 - tid) * EL::SIZE);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (steps * U * NT + u * NT < rest) last[u] = words[steps * U * NT + u * NT];
  auto load = [&](int s, u32x4* to) {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = words[s * (U * NT) + u * NT];
  };
  auto add = [&](const u32x4* from) {
    float e[U * EL::N];
#pragma unroll
    for (int u = 0; u < U; ++u) EL::widen(from[u], e + u * EL::N);
    sum.add<U * EL::N>(e, c);
  };
  if (steps > 0) {
    load(0, w);
#pragma unroll 2
    for (int s = 1; s < steps; ++s) {
      load(s, next);
      add(w);
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = next[u];
    }
    add(w);
  }
  if (edges && tid < 16) sum.add<2>(edge, c);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (steps * U * NT + u * NT < rest) {
      float e[EL::N];
      EL::widen(last[u], e);
      sum.add<EL::N>(e, c);
    }
  }
  const float R = group_max<NT>(sum.R);
  sum.raise(R);
  return {R, group_total<NT>(sum.s)};
}

// A row's results from its sum.
template <int DT, int NT>
__device__ __forceinline__ void finish_row(const char* x, int vocab, int y, float scale, Sum sum, float* logp, float* lse,
                                           int* bad_flag) {
  using EL = Elem<DT>;
  const int tid = threadIdx.x & (NT - 1);
  const float c = scale * LOG2E;
  double ref = (double)sum.R / (double)c;  // the sum is of exp(scale (x - ref))
  if (!(sum.R > LEAST && sum.R < -LEAST)) {
    // No power above -2^24, or one beyond 2^24: once more, with differences from the largest logit.
    float m = -__builtin_inff();
    for (int j = tid; j < vocab; j += NT) m = fmaxf(m, EL::load(x + (size_t)j * EL::SIZE));
    m = group_max<NT>(m);
    float s = 0.f;
    for (int j = tid; j < vocab; j += NT) s += __builtin_amdgcn_exp2f((EL::load(x + (size_t)j * EL::SIZE) - m) * c);
    sum.s = group_total<NT>(s);
    ref = m;
  }
  if (tid != 0) return;
  const double ls = log((double)sum.s);
  if (lse) *lse = (float)((double)scale * ref + ls);
  if (y < vocab) {
    *logp = (float)((double)scale * ((double)EL::load(x + (size_t)y * EL::SIZE) - ref) - ls);
  } else {
    *logp = __builtin_nanf("");
    if (bad_flag) *bad_flag = 1;
  }
}

struct RowArgs {
  const char* X;
  long long ld;
  const int* labels;
  float scale;
  float *logp, *lse;
  int* bad_flag;
  int T, vocab;
  unsigned rows;
  int parts;
  float2* part;
};

__device__ __forceinline__ int row_label(const RowArgs& a, unsigned row, bool write) {
  const int y = a.labels[row % (unsigned)a.T];
  if (y < 0 && write) {
    a.logp[row] = 0.f;
    if (a.lse) a.lse[row] = 0.f;
  }
  return y;
}

// NT threads per row: a wave each of four rows in a workgroup, or the workgroup.  One pass over the logits, which bounds it: 6.2
// TB/s of reads at 8192 rows of 151851 bf16 (277 us) and 8000 of 32000 fp32 (113); 6.6 vector instructions a
// logit, of which the exponential costs four, would take 210 of the 277.
template <int DT, int NT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_token_logprob(RowArgs a) {
  const unsigned block = blockIdx.y * gridDim.x + blockIdx.x, row = NT < 256 ? block * 4 + (threadIdx.x >> 6) : block;
  if (row >= a.rows) return;
  const int y = row_label(a, row, (threadIdx.x & (NT - 1)) == 0);
  if (y < 0) return;
  const char* x = a.X + (size_t)row * a.ld * Elem<DT>::SIZE;
  const RowWords r = row_words<DT>(x, a.vocab);
  const Sum sum = row_sum<DT, NT>(x, r, a.vocab, 0, r.words, true, a.scale * LOG2E);
  finish_row<DT, NT>(x, a.vocab, y, a.scale, sum, a.logp + row, a.lse ? a.lse + row : nullptr, a.bad_flag);
}

// A part of a row per workgroup, and the parts' join, a wave per row: 3.9 and 3.2 us for 5 rows of 151936 bf16.
template <int DT>
__global__ __launch_bounds__(256) void k_token_logprob_part(RowArgs a) {
  const unsigned row = blockIdx.y;
  const int p = blockIdx.x;
  if (row_label(a, row, false) < 0) return;
  const char* x = a.X + (size_t)row * a.ld * Elem<DT>::SIZE;
  const RowWords r = row_words<DT>(x, a.vocab);
  const int each = (r.words + a.parts - 1) / a.parts, lo = min(p * each, r.words), hi = min(lo + each, r.words);
  const Sum sum = row_sum<DT, 256>(x, r, a.vocab, lo, hi, p == 0, a.scale * LOG2E);
  if (threadIdx.x == 0) a.part[(size_t)row * a.parts + p] = make_float2(sum.R, sum.s);
}

template <int DT>
__global__ __launch_bounds__(64) void k_token_logprob_join(RowArgs a) {
  const unsigned row = blockIdx.x;
  const int y = row_label(a, row, threadIdx.x == 0);
  if (y < 0) return;
  Sum sum = {LEAST, 0.f};
  if ((int)threadIdx.x < a.parts) {
    const float2 v = a.part[(size_t)row * a.parts + threadIdx.x];
    sum = {v.x, v.y};
  }
  const float R = group_max<64>(sum.R);
  sum.raise(R);
  sum = {R, group_total<64>(sum.s)};
  finish_row<DT, 64>(a.X + (size_t)row * a.ld * Elem<DT>::SIZE, a.vocab, y, a.scale, sum, a.logp + row,
                     a.lse ? a.lse + row : nullptr, a.bad_flag);
}

// dx = c g ([j = y] - exp(c x - lse)), word by word: 256 threads take 2 words each of a row; the first workgroup of a row also
// its elements before and behind the words.  Reads and writes bound it: 8192 rows of 50272 fp16, 5733 of them counted, 247 us, 5.7
// TB/s; with 1 word a thread 284, with 4 252 (16000 rows of 6000 fp32 128, 114, 142), with loads under their bounds checks 258.
constexpr int BACK_U = 2;
template <int DT>
__global__ __launch_bounds__(256) void k_token_logprob_backward(const char* X, long long ld, const int* __restrict__ labels,
                                                                float scale, const float* __restrict__ lse,
                                                                const float* __restrict__ logp,
                                                                const float* __restrict__ g, char* dX, long long ldo,
                                                                int* bad_flag, int T, int vocab, unsigned rows) {
  using EL = Elem<DT>;
  const int tid = threadIdx.x;
  for (unsigned row = blockIdx.y; row < rows; row += gridDim.y) {
    const int y = labels[row % (unsigned)T];
    const char* x = X + (size_t)row * ld * EL::SIZE;
    char* out = dX + (size_t)row * ldo * EL::SIZE;
    float up = 0.f, z = 0.f, ref = 0.f;
    if (y >= vocab) {
      up = __builtin_nanf("");
      if (bad_flag && blockIdx.x == 0 && tid == 0) *bad_flag = 1;
    } else if (y >= 0) {
      up = scale * g[row];
      z = lse[row];
      // The smaller of the two has the smaller rounding: c (x - x_y) + logp is c x - lse.
      if (logp && fabsf(logp[row]) < fabsf(z)) {
        z = -logp[row];
        ref = EL::load(x + (size_t)y * EL::SIZE);
      }
    }
    auto grad = [&](float v, bool hit) {
      const float p = __builtin_amdgcn_exp2f(fmaf(v - ref, scale, -z) * LOG2E);
      return up * ((hit ? 1.f : 0.f) - p);
    };
    // Rows that begin elsewhere in a word, element by element: 8192 rows of 151851 bf16 1805 us, where words take 821.
    if (((uintptr_t)x ^ (uintptr_t)out) & 15) {
#pragma unroll 1
      for (int k = 0; k < BACK_U * EL::N; ++k) {
        const int j = (blockIdx.x * BACK_U * EL::N + k) * 256 + tid;
        if (j < vocab) EL::store(out + (size_t)j * EL::SIZE, y < 0 ? 0.f : grad(EL::load(x + (size_t)j * EL::SIZE), j == y));
      }
      continue;
    }
    const RowWords r = row_words<DT>(x, vocab);
    if (blockIdx.x == 0 && tid < 16) {
      const int j = tid < 8 ? (tid < r.head ? tid : -1) : (tid - 8 < r.tail ? vocab - 1 - (tid - 8) : -1);
      if (j >= 0) EL::store(out + (size_t)j * EL::SIZE, y < 0 ? 0.f : grad(EL::load(x + (size_t)j * EL::SIZE), j == y));
    }
    const u32x4* words = (const u32x4*)(x + r.head * EL::SIZE);
    u32x4* to = (u32x4*)(out + r.head * EL::SIZE);
    const int i0 = blockIdx.x * (256 * BACK_U) + tid;
    if (y < 0) {
#pragma unroll
      for (int u = 0; u < BACK_U; ++u)
        if (i0 + u * 256 < r.words) to[i0 + u * 256] = (u32x4){0, 0, 0, 0};
      continue;
    }
    if (i0 >= r.words) continue;
    u32x4 w[BACK_U];
#pragma unroll
    for (int u = 0; u < BACK_U; ++u) w[u] = words[min(i0 + u * 256, r.words - 1)];
#pragma unroll
    for (int u = 0; u < BACK_U; ++u) {
      const int i = i0 + u * 256;
      if (i >= r.words) break;
      float e[EL::N];
      EL::widen(w[u], e);
      const int hit = y - r.head - i * EL::N;
      if ((unsigned)hit < (unsigned)EL::N) {
#pragma unroll
        for (int k = 0; k < EL::N; ++k) e[k] = grad(e[k], k == hit);
      } else {
#pragma unroll
        for (int k = 0; k < EL::N; ++k) e[k] = grad(e[k], false);
      }
      to[i] = EL::narrow(e);
    }
  }
}

}  // namespace

int zo_token_logprob_launch(int nblk, int T, int vocab, int dtype, const void* X, long long ld, const int* labels, float scale,
                            float* logp, float* lse, int* bad_flag, void* ws, hipStream_t stream, size_t* ws_needed) {
  const unsigned rows = (unsigned)nblk * (unsigned)T;
  const long long bytes = (long long)vocab * (dtype == ZO_F32 ? 4 : 2);
  RowArgs a = {(const char*)X, ld, labels, scale, logp, lse, bad_flag, T, vocab, rows, 1, (float2*)ws};
  // Few long rows are split: a workgroup's exponentials alone take 8 us for 151936 logits.  us of the kernels, whole and split, bf16:
  // 5 rows of 151936 10.7 and 7.3, 61 rows 11.5 and 9.7, 120 rows 11.7 and 11.6; one row of 50272 6.3 and 6.9, 60 rows 6.8 and 7.8.
  // (In graphs of one after another 5, 61, 120 and 256 rows take 6.2, 8.0, 11.0 and 15.6.)
  if (rows <= 64 && bytes >= 262144) a.parts = (int)min(min(64LL, (bytes + 16383) / 16384), 512LL / rows);
  if (ws_needed) {
    *ws_needed = a.parts > 1 ? zo_align256((size_t)rows * a.parts * sizeof(float2)) : 0;
    return ZO_OK;
  }
  auto go = [&](auto k, int threads, unsigned per) {
    // A grid's x dimension holds fewer than 2^32 threads.
    const unsigned n = rows / per + (rows % per != 0), x = n < (1u << 20) ? n : 1u << 20;
    hipLaunchKernelGGL(k, dim3(x, (n + x - 1) / x), dim3(threads), 0, stream, a);
    return zo_hip_status(hipGetLastError(), "k_token_logprob");
  };
  auto of = [&](auto part, auto join, auto wave, auto small, auto large) {
    if (a.parts > 1) {
      hipLaunchKernelGGL(part, dim3(a.parts, rows), dim3(256), 0, stream, a);
      const int st = zo_hip_status(hipGetLastError(), "k_token_logprob_part");
      if (st != ZO_OK) return st;
      hipLaunchKernelGGL(join, dim3(rows), dim3(64), 0, stream, a);
      return zo_hip_status(hipGetLastError(), "k_token_logprob_join");
    }
    // us with a wave, 256 and 1024 threads a row: 64000 rows of 1500 fp32 51, 83, 284; 32000 of 6000 bf16 52, 59, 159; of 12000
    // 97, 96, 193; 2400 of 6000 9.0, 8.6, 15.1; 16000 of 40000 159, 152, 166; 12000 of 50272 154, 143, 144; of 65000 198, 186, 183;
    // of 25000 fp32 148, 142, 136; 5600 of 151851 bf16 290, 299, 279.
    return bytes <= 12288 && rows >= 4096 ? go(wave, 256, 4) : bytes <= 98304 ? go(small, 256, 1) : go(large, 1024, 1);
  };
  auto kernels = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    return of(k_token_logprob_part<DT>, k_token_logprob_join<DT>, k_token_logprob<DT, 64>, k_token_logprob<DT, 256>,
              k_token_logprob<DT, 1024>);
  };
  return dtype == ZO_F32 ? kernels(std::integral_constant<int, ZO_F32>())
         : dtype == ZO_BF16 ? kernels(std::integral_constant<int, ZO_BF16>())
                            : kernels(std::integral_constant<int, ZO_F16>());
}

int zo_token_logprob_backward_launch(int nblk, int T, int vocab, int dtype, const void* X, long long ld, const int* labels,
                                     float scale, const float* lse, const float* logp, const float* g, void* dX, long long ldo,
                                     int* bad_flag, hipStream_t stream) {
  const unsigned rows = (unsigned)nblk * (unsigned)T;
  const int per = 256 * BACK_U * (dtype == ZO_F32 ? 4 : 8);
  const dim3 grid((unsigned)((vocab + (long long)per - 1) / per), rows < 65535 ? rows : 65535);
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, grid, dim3(256), 0, stream, (const char*)X, ld, labels, scale, lse, logp, g, (char*)dX, ldo, bad_flag, T,
                       vocab, rows);
  };
  if (dtype == ZO_F32) go(k_token_logprob_backward<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_token_logprob_backward<ZO_BF16>);
  else go(k_token_logprob_backward<ZO_F16>);
  return zo_hip_status(hipGetLastError(), "k_token_logprob_backward");
}
