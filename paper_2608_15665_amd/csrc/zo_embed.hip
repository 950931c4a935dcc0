// Embedding lookup and the table's gradient by sorted tokens.
#include "zo_attn.h"

namespace {

constexpr int SORT_TILE = 2048;    // tokens per sorting workgroup: 8 waves of 4 x 64
constexpr int SORT_WAVES = 8;
constexpr int MAX_DIGITS = 512;    // 9 bits a pass: two passes sort any vocabulary below 2^18
constexpr int CHUNK = 32;          // sorted positions that one wave sums

// n workgroups of 256 threads, in rows of 2^22 where there are more: a grid's x dimension holds fewer than 2^32 threads.
dim3 grid_of(long long n) {
  if (n < (1LL << 22)) return dim3((unsigned)n);
  return dim3(1u << 22, (unsigned)((n + (1LL << 22) - 1) >> 22));
}
__device__ __forceinline__ long long block_of() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------- lookup
template <int DT>
__global__ __launch_bounds__(256) void k_embedding(const int* __restrict__ ids, const void* __restrict__ E, float scale,
                                                   void* __restrict__ H, int* bad_flag, long long rows, int vocab, int d) {
  const int per = d / 8;
  const long long i = block_of() * 256 + threadIdx.x;
  const long long row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 8;
  const int id = ids[row];
  float v[8];
  if (id >= 0 && id < vocab) {
    load8<DT>(E, (size_t)id * d + c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
  } else {
    const float fill = id < 0 ? 0.f : __builtin_nanf("");
    if (id >= 0 && bad_flag && c == 0) *bad_flag = 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fill;
  }
  store8<DT>(H, (size_t)row * d + c, v);
}

// ---------------------------------------------------------------- sorting
// Stable radix sort of the pairs (token, row), least digit first.  Tokens that have no row of the table are taken
// as `vocab` and so come last.
struct SortPlan {
  int n, vocab, ntiles, passes, shift[4], mask[4];
};

__device__ __forceinline__ int token_key(const int* ids, int i, int vocab, int* bad_flag) {
  const int id = ids[i];
  if (id >= vocab && bad_flag) *bad_flag = 1;
  return (unsigned)id < (unsigned)vocab ? id : vocab;
}

// Digit counts of a tile for the first pass; clears the counts of the later ones.
__global__ __launch_bounds__(512) void k_sort_count(const int* __restrict__ ids, SortPlan p, int* hist, int* bad_flag) {
  __shared__ int cnt[MAX_DIGITS];
  const int t = threadIdx.x;
  cnt[t] = 0;
  __syncthreads();
  for (int k = 0; k < SORT_TILE / 512; ++k) {
    const int i = blockIdx.x * SORT_TILE + k * 512 + t;
    if (i < p.n) atomicAdd(&cnt[token_key(ids, i, p.vocab, bad_flag) & p.mask[0]], 1);
  }
  __syncthreads();
  hist[(size_t)blockIdx.x * MAX_DIGITS + t] = cnt[t];
  for (int q = 1; q < p.passes; ++q) hist[((size_t)q * p.ntiles + blockIdx.x) * MAX_DIGITS + t] = 0;
}

// One pass: a tile's items to their places among all, and the next pass's counts where they land (integer counts:
// their order does not matter).
__global__ __launch_bounds__(512) void k_sort_scatter(const int* __restrict__ ids, SortPlan p, int pass, const int* hist,
                                                      int* next_hist, const int* key_in, const int* row_in, int* key_out,
                                                      int* row_out) {
  __shared__ int cnt[SORT_WAVES][MAX_DIGITS];
  __shared__ int wsum[SORT_WAVES];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  // Items of this digit in all tiles, and in the tiles before this one.
  int before = 0, total = 0;
  for (int j = 0; j < p.ntiles; ++j) {
    const int c = hist[(size_t)j * MAX_DIGITS + t];
    before += j < (int)blockIdx.x ? c : 0;
    total += c;
  }
#pragma unroll
  for (int j = 0; j < SORT_WAVES; ++j) cnt[j][t] = 0;
  int sum = total;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(sum, off, 64);
    if (lane >= off) sum += v;
  }
  if (lane == 63) wsum[w] = sum;
  __syncthreads();
  int base = sum - total + before;
  for (int j = 0; j < w; ++j) base += wsum[j];
  // Rank of each item among those of its wave with its digit: earlier items of 64 by a ballot per bit, earlier groups
  // of 64 by a running count.
  int key[4], row[4], rank[4];
  volatile int* mine = cnt[w];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = blockIdx.x * SORT_TILE + w * 256 + k * 64 + lane;
    const bool on = i < p.n;
    key[k] = !on ? 0 : pass == 0 ? token_key(ids, i, p.vocab, nullptr) : key_in[i];
    row[k] = !on ? -1 : pass == 0 ? i : row_in[i];
    const int dig = (key[k] >> p.shift[pass]) & p.mask[pass];
    unsigned long long same = __ballot(on);
#pragma unroll
    for (int b = 0; b < 9; ++b) {
      const unsigned long long bits = __ballot((dig >> b) & 1);
      same &= (dig >> b) & 1 ? bits : ~bits;
    }
    const int prior = mine[dig];
    __builtin_amdgcn_wave_barrier();
    const int ahead = __popcll(same & ((1ull << lane) - 1));
    rank[k] = prior + ahead;
    if (on && ahead == 0) mine[dig] = prior + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < SORT_WAVES; ++j) {
    const int c = cnt[j][t];
    cnt[j][t] = base;
    base += c;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (row[k] < 0) continue;
    const int to = cnt[w][(key[k] >> p.shift[pass]) & p.mask[pass]] + rank[k];
    key_out[to] = key[k];
    row_out[to] = row[k];
    if (next_hist)
      atomicAdd(&next_hist[(size_t)(to / SORT_TILE) * MAX_DIGITS + ((key[k] >> p.shift[pass + 1]) & p.mask[pass + 1])], 1);
  }
}

// ---------------------------------------------------------------- sums
__global__ __launch_bounds__(256) void k_fill_zero(u32x4* p, long long n) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256)
    p[i] = (u32x4){0, 0, 0, 0};
}

template <int OT>
__device__ __forceinline__ void put_row(void* dE, size_t at, const float* s, float scale, int add) {
  float v[8];
  if (add) {
    load8<OT>(dE, at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(scale, s[e], v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scale * s[e];
  }
  store8<OT>(dE, at, v);
}

// A wave sums 512 columns of CHUNK sorted positions.  Tokens that lie whole in them are written; the sums of one that
// came in from the positions before, or goes on behind, are kept: part[2 chunk] and part[2 chunk + 1].
template <int DT, int OT>
__global__ __launch_bounds__(256) void k_embed_sum(const int* __restrict__ key, const int* __restrict__ row, int n, int vocab,
                                                   int d, const void* __restrict__ dH, float scale, void* dE, int add,
                                                   float* part, int nchunk, int nslab) {
  const long long wave = block_of() * 4 + (threadIdx.x >> 6);
  const int chunk = (int)(wave / nslab), c = (int)(wave % nslab) * 512 + (threadIdx.x & 63) * 8;
  if (chunk >= nchunk || c >= d) return;
  const int i0 = chunk * CHUNK, i1 = min(i0 + CHUNK, n);
  bool inside = i0 == 0 || key[i0 - 1] != key[i0];  // the running token began in this chunk
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = i0; i < i1; ++i) {
    const int k = key[i];
    if (k >= vocab) return;
    float v[8];
    load8<DT>(dH, (size_t)row[i] * d + c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
    const int next = i + 1 < n ? key[i + 1] : vocab;
    if (next == k && i + 1 < i1) continue;
    if (next != k && inside)
      put_row<OT>(dE, (size_t)k * d + c, s, scale, add);
    else
      store8<ZO_F32>(part, ((size_t)2 * chunk + (inside ? 1 : 0)) * d + c, s);
    inside = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
  }
}

// Joins the sums of each token that lies in more than one chunk: the wave of the chunk where it begins adds them in order.
template <int OT>
__global__ __launch_bounds__(256) void k_embed_join(const int* __restrict__ key, int n, int vocab, int d, float scale, void* dE,
                                                    int add, const float* part, int nchunk, int nslab) {
  const long long wave = block_of() * 4 + (threadIdx.x >> 6);
  const int chunk = (int)(wave / nslab), c = (int)(wave % nslab) * 512 + (threadIdx.x & 63) * 8;
  if (chunk >= nchunk - 1 || c >= d) return;
  const int i0 = chunk * CHUNK, last = i0 + CHUNK - 1, k = key[last];
  if (k >= vocab || key[last + 1] != k) return;
  if (key[i0] == k && i0 > 0 && key[i0 - 1] == k) return;  // it began earlier
  float s[8], v[8];
  load8<ZO_F32>(part, ((size_t)2 * chunk + 1) * d + c, s);
  for (int j = chunk + 1; j < nchunk && key[j * CHUNK] == k; ++j) {
    load8<ZO_F32>(part, (size_t)2 * j * d + c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
  put_row<OT>(dE, (size_t)k * d + c, s, scale, add);
}

SortPlan sort_plan(long long n, int vocab) {
  SortPlan p = {};
  p.n = (int)n;
  p.vocab = vocab;
  p.ntiles = (int)((n + SORT_TILE - 1) / SORT_TILE);
  int bits = 1;
  while (bits < 31 && (vocab >> bits)) ++bits;  // keys 0 .. vocab
  p.passes = (bits + 8) / 9;
  const int w = (bits + p.passes - 1) / p.passes;
  for (int q = 0; q < p.passes; ++q) {
    p.shift[q] = q * w;
    p.mask[q] = (1 << w) - 1;
  }
  return p;
}

}  // namespace

int zo_embedding_launch(long long rows, int vocab, int d, int dtype, const int* ids, const void* E, float scale, void* H,
                        int* bad_flag, hipStream_t stream) {
  const dim3 grid = grid_of((rows * (d / 8) + 255) / 256);
  auto go = [&](auto k) { hipLaunchKernelGGL(k, grid, dim3(256), 0, stream, ids, E, scale, H, bad_flag, rows, vocab, d); };
  if (dtype == ZO_F32) go(k_embedding<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_embedding<ZO_BF16>);
  else go(k_embedding<ZO_F16>);
  return zo_hip_status(hipGetLastError(), "k_embedding");
}

int zo_embedding_backward_launch(long long rows, int vocab, int d, int dtype, const int* ids, const void* dH, float scale,
                                 int out_dtype, void* dE, int accumulate, int* bad_flag, void* ws, hipStream_t stream,
                                 size_t* ws_needed) {
  const SortPlan p = sort_plan(rows, vocab);
  const int nchunk = (p.n + CHUNK - 1) / CHUNK, nslab = (d + 511) / 512;
  WsCarver w(ws);
  int* hist = (int*)w.take((size_t)p.passes * p.ntiles * MAX_DIGITS * sizeof(int));
  int* key[2] = {(int*)w.take((size_t)p.n * 4), (int*)w.take((size_t)p.n * 4)};
  int* row[2] = {(int*)w.take((size_t)p.n * 4), (int*)w.take((size_t)p.n * 4)};
  float* part = (float*)w.take((size_t)2 * nchunk * d * sizeof(float));
  if (ws_needed) {
    *ws_needed = rows ? w.off : 0;
    return ZO_OK;
  }
  if (!accumulate) {
    const long long words = (long long)vocab * d / (out_dtype == ZO_F32 ? 4 : 8);
    hipLaunchKernelGGL(k_fill_zero, dim3((unsigned)min((words + 1023) / 1024, 8192LL)), dim3(256), 0, stream, (u32x4*)dE, words);
    const int st = zo_hip_status(hipGetLastError(), "k_fill_zero");
    if (st != ZO_OK || rows == 0) return st;
  }
  if (rows == 0) return ZO_OK;
  hipLaunchKernelGGL(k_sort_count, dim3(p.ntiles), dim3(512), 0, stream, ids, p, hist, bad_flag);
  int st = zo_hip_status(hipGetLastError(), "k_sort_count");
  for (int q = 0; q < p.passes && st == ZO_OK; ++q) {
    const size_t step = (size_t)p.ntiles * MAX_DIGITS;
    hipLaunchKernelGGL(k_sort_scatter, dim3(p.ntiles), dim3(512), 0, stream, ids, p, q, hist + q * step,
                       q + 1 < p.passes ? hist + (q + 1) * step : nullptr, key[(q + 1) & 1], row[(q + 1) & 1], key[q & 1],
                       row[q & 1]);
    st = zo_hip_status(hipGetLastError(), "k_sort_scatter");
  }
  if (st != ZO_OK) return st;
  const int *skey = key[(p.passes - 1) & 1], *srow = row[(p.passes - 1) & 1];
  const dim3 grid = grid_of(((long long)nchunk * nslab + 3) / 4);
  auto go = [&](auto sum, auto join) {
    hipLaunchKernelGGL(sum, grid, dim3(256), 0, stream, skey, srow, p.n, vocab, d, dH, scale, dE, accumulate, part, nchunk, nslab);
    st = zo_hip_status(hipGetLastError(), "k_embed_sum");
    if (st != ZO_OK || nchunk == 1) return;
    hipLaunchKernelGGL(join, grid, dim3(256), 0, stream, skey, p.n, vocab, d, scale, dE, accumulate, part, nchunk, nslab);
    st = zo_hip_status(hipGetLastError(), "k_embed_join");
  };
  if (dtype == ZO_F32) go(k_embed_sum<ZO_F32, ZO_F32>, k_embed_join<ZO_F32>);
  else if (dtype == ZO_BF16 && out_dtype == ZO_F32) go(k_embed_sum<ZO_BF16, ZO_F32>, k_embed_join<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_embed_sum<ZO_BF16, ZO_BF16>, k_embed_join<ZO_BF16>);
  else if (out_dtype == ZO_F32) go(k_embed_sum<ZO_F16, ZO_F32>, k_embed_join<ZO_F32>);
  else go(k_embed_sum<ZO_F16, ZO_F16>, k_embed_join<ZO_F16>);
  return st;
}
