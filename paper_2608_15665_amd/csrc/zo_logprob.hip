// Log-probabilities of labelled tokens over the vocabulary, and the logits' gradient.
#include "zo_internal.h"

namespace {

template <int DT>
__device__ __forceinline__ float logit(const void* X, size_t i) {
  if constexpr (DT == ZO_F32) return ((const float*)X)[i];
  else if constexpr (DT == ZO_BF16) return bf16_to_f32(((const bf16_t*)X)[i]);
  else return f16_to_f32(((const uint16_t*)X)[i]);
}

constexpr float LOG2E = 1.4426950408889634f;

// A workgroup per row: the largest logit, then the sum relative to it.
template <int DT>
__global__ __launch_bounds__(256) void k_token_logprob(const void* __restrict__ X, long long ld, const int* __restrict__ labels,
                                                       float scale, float* logp, float* lse, int* bad_flag, int T, int vocab,
                                                       long long rows) {
  __shared__ float red[8];
  for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
    const int y = labels[row % T];
    if (y < 0) {
      if (threadIdx.x == 0) {
        logp[row] = 0.f;
        if (lse) lse[row] = 0.f;
      }
      continue;
    }
    const size_t at = (size_t)row * ld;
    float m = -__builtin_inff();
    for (int j = threadIdx.x; j < vocab; j += 256) m = fmaxf(m, logit<DT>(X, at + j));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float s = 0.f;
    for (int j = threadIdx.x; j < vocab; j += 256)
      s += __builtin_amdgcn_exp2f((logit<DT>(X, at + j) - m) * (scale * LOG2E));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    if ((threadIdx.x & 63) == 0) red[4 + (threadIdx.x >> 6)] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      const double ls = log((double)((red[4] + red[5]) + (red[6] + red[7])));
      if (lse) lse[row] = (float)((double)scale * m + ls);
      if (y < vocab) {
        logp[row] = (float)((double)scale * ((double)logit<DT>(X, at + y) - (double)m) - ls);
      } else {
        logp[row] = __builtin_nanf("");
        if (bad_flag) *bad_flag = 1;
      }
    }
  }
}

template <int DT>
__global__ __launch_bounds__(256) void k_token_logprob_backward(const void* X, long long ld, const int* __restrict__ labels,
                                                                float scale, const float* __restrict__ lse,
                                                                const float* __restrict__ g, void* dX, long long ldo,
                                                                int* bad_flag, int T, int vocab, long long rows) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= vocab) return;
  for (long long row = blockIdx.y; row < rows; row += gridDim.y) {
    const int y = labels[row % T];
    float v = 0.f;
    if (y >= vocab) {
      v = __builtin_nanf("");
      if (bad_flag && j == 0) *bad_flag = 1;
    } else if (y >= 0) {
      const float p = __builtin_amdgcn_exp2f(fmaf(logit<DT>(X, (size_t)row * ld + j), scale, -lse[row]) * LOG2E);
      v = scale * g[row] * ((j == y ? 1.f : 0.f) - p);
    }
    const size_t to = (size_t)row * ldo + j;
    if constexpr (DT == ZO_F32) ((float*)dX)[to] = v;
    else if constexpr (DT == ZO_BF16) ((bf16_t*)dX)[to] = f32_to_bf16(v);
    else ((uint16_t*)dX)[to] = f32_to_f16(v);
  }
}

}  // namespace

int zo_token_logprob_launch(int nblk, int T, int vocab, int dtype, const void* X, long long ld, const int* labels, float scale,
                            float* logp, float* lse, int* bad_flag, hipStream_t stream) {
  const long long rows = (long long)nblk * T;
  const dim3 grid((unsigned)(rows < (1 << 20) ? rows : (1 << 20)));
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, grid, dim3(256), 0, stream, X, ld, labels, scale, logp, lse, bad_flag, T, vocab, rows);
  };
  if (dtype == ZO_F32) go(k_token_logprob<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_token_logprob<ZO_BF16>);
  else go(k_token_logprob<ZO_F16>);
  return zo_hip_status(hipGetLastError(), "k_token_logprob");
}

int zo_token_logprob_backward_launch(int nblk, int T, int vocab, int dtype, const void* X, long long ld, const int* labels,
                                     float scale, const float* lse, const float* g, void* dX, long long ldo, int* bad_flag,
                                     hipStream_t stream) {
  const long long rows = (long long)nblk * T;
  const dim3 grid((unsigned)((vocab + 255LL) / 256), (unsigned)(rows < 65535 ? rows : 65535));
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, grid, dim3(256), 0, stream, X, ld, labels, scale, lse, g, dX, ldo, bad_flag, T, vocab, rows);
  };
  if (dtype == ZO_F32) go(k_token_logprob_backward<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_token_logprob_backward<ZO_BF16>);
  else go(k_token_logprob_backward<ZO_F16>);
  return zo_hip_status(hipGetLastError(), "k_token_logprob_backward");
}
