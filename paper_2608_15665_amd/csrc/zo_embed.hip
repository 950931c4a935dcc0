// Embedding lookup and the table's gradient by sorted tokens.
#include "zo_attn.h"

#include <type_traits>

namespace {

constexpr int SORT_WAVES = 8, SORT_TILE = SORT_WAVES * 256;  // of a sorting workgroup, and its tokens
constexpr int DIGITS = 512;     // 9 bits a pass: two passes sort any vocabulary below 2^18
constexpr int SORT_ONE = 8192;  // tokens that one workgroup of 16 waves sorts (20 us; in tiles 4 launches, no faster)
// Tokens that are compared rather than sorted.  us, compared and sorted, adding rows of 4096 bf16 to fp32: 256 tokens of a
// text 5.8 and 18.8, 500 8.0 and 19.3, 1000 15.9 and 22.7; 500 times the same token 42 and 15, 1000 times 116 and 15.
constexpr int FEW = 512;
constexpr int JOIN_WAVES = 8, JOIN_ALONE = 16;

// n workgroups of 256 threads, in rows of 2^22 where there are more: a grid's x dimension holds fewer than 2^32 threads.
dim3 grid_of(long long n) {
  if (n < (1LL << 22)) return dim3((unsigned)n);
  return dim3(1u << 22, (unsigned)((n + (1LL << 22) - 1) >> 22));
}
__device__ __forceinline__ long long block_of() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------- lookup
// 16-byte words of a row that a wave takes at a time: all are on their way before the first is stored.
constexpr int SPAN = 2;

template <int DT>
__device__ __forceinline__ u32x4 scaled(const u32x4& w, float scale) {
  u32x4 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == ZO_F32) r[k] = __float_as_uint(__uint_as_float(w[k]) * scale);
    else if constexpr (DT == ZO_BF16)
      r[k] = pack_bf16x2(__uint_as_float(w[k] << 16) * scale, __uint_as_float(w[k] & 0xffff0000u) * scale);
    else r[k] = pack_f16x2(f16_to_f32((uint16_t)w[k]) * scale, f16_to_f32((uint16_t)(w[k] >> 16)) * scale);
  }
  return r;
}

// A wave takes 64 SPAN words of the result, whatever rows they lie in.  The result is stored past the caches, which then
// keep the table's frequent rows: 65536 rows of 4096 bf16 170 us without, 114 with (5.7 TB/s); 1024 rows 5.4 and 5.0.
template <int DT>
__global__ __launch_bounds__(256) void k_embedding(const int* __restrict__ ids, const u32x4* __restrict__ E, float scale,
                                                   u32x4* __restrict__ H, int* bad_flag, long long total, int vocab, int words) {
  const long long first = (block_of() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (64 * SPAN);
  if (first >= total) return;
  const int lane = threadIdx.x & 63;
  const long long row0 = first / words;
  const int off = (int)(first - row0 * words);
  const float inv = 1.f / (float)words;
  u32x4 w[SPAN];
  int id[SPAN], c[SPAN];
#pragma unroll
  for (int u = 0; u < SPAN; ++u) {
    const int o = off + min(u * 64 + lane, (int)min(total - 1 - first, 64LL * SPAN));  // below words + 64 SPAN < 2^19:
    int k = (int)((float)o * inv);                                                     // the quotient is at most one off
    k += (o - k * words >= words) - (o < k * words);
    c[u] = o - k * words;
    id[u] = ids[row0 + k];
  }
  // No load hangs on a condition: it would wait for the ones before it.
#pragma unroll
  for (int u = 0; u < SPAN; ++u) w[u] = E[(size_t)min(max(id[u], 0), vocab - 1) * words + c[u]];
#pragma unroll
  for (int u = 0; u < SPAN; ++u) {
    u32x4 v = scaled<DT>(w[u], scale);
    if ((unsigned)id[u] >= (unsigned)vocab) {
      const uint32_t fill = id[u] < 0 ? 0u : DT == ZO_F32 ? 0x7fc00000u : DT == ZO_BF16 ? 0x7fc07fc0u : 0x7e007e00u;  // NaN
      v = (u32x4){fill, fill, fill, fill};
      if (id[u] >= 0 && bad_flag && c[u] == 0) *bad_flag = 1;
    }
    if (first + u * 64 + lane < total) __builtin_nontemporal_store(v, H + first + u * 64 + lane);
  }
}

// ---------------------------------------------------------------- sorting
// Stable radix sort of the pairs (token, row), least digit first.  Tokens that have no row of the table are taken as
// `vocab` and so come last.  While few workgroups sort, the others of the launch clear their share of a dense gradient:
// the sorting of 8192 tokens, 20 us, is hidden behind the 80 that clearing 50272 x 5120 bf16 takes (6.4 TB/s).
struct SortPlan {
  int n, vocab, ntiles, passes, shift[4], mask[4];
};
struct Fill {
  u32x4* p;
  long long lo, hi;  // words to clear in this launch
  int sorters;       // the launch's first workgroups, which sort
};

__device__ __forceinline__ bool clears(const Fill& f) {
  if ((int)blockIdx.x < f.sorters) return false;
  const long long step = (long long)(gridDim.x - f.sorters) * blockDim.x;
  for (long long i = f.lo + (long long)(blockIdx.x - f.sorters) * blockDim.x + threadIdx.x; i < f.hi; i += step)
    f.p[i] = (u32x4){0, 0, 0, 0};
  return true;
}

__device__ __forceinline__ int token_key(const int* ids, int i, int vocab, int* bad_flag) {
  const int id = ids[i];
  if (id >= vocab && bad_flag) *bad_flag = 1;
  return (unsigned)id < (unsigned)vocab ? id : vocab;
}

// Where an item stands among those of its wave with its digit: earlier ones of its 64 by a ballot per bit, earlier
// groups of 64 by a running count.
template <typename C>
__device__ __forceinline__ int wave_rank(volatile C* count, int digit, bool on) {
  unsigned long long same = __ballot(on);
#pragma unroll
  for (int b = 0; b < 9; ++b) {
    const unsigned long long bits = __ballot((digit >> b) & 1);
    same &= (digit >> b) & 1 ? bits : ~bits;
  }
  const int prior = count[digit], ahead = __popcll(same & ((1ull << (threadIdx.x & 63)) - 1));
  __builtin_amdgcn_wave_barrier();
  if (on && ahead == 0) count[digit] = (C)(prior + __popcll(same));
  __builtin_amdgcn_wave_barrier();
  return prior + ahead;
}

// Exclusive sums over 512 digits, one per thread of the first eight waves.
__device__ __forceinline__ int digits_before(int count, int* wsum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int sum = count;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(sum, off, 64);
    if (lane >= off) sum += v;
  }
  if (lane == 63 && w < 8) wsum[w] = sum;
  __syncthreads();
  int base = sum - count;
  for (int j = 0; j < w && j < 8; ++j) base += wsum[j];
  return base;
}

// The whole sort in one workgroup: (token << 13 | row) in LDS from pass to pass.  Ballots and LDS round trips in a row bound it, 6 us
// for 300 tokens, 20 for 8192.
__global__ __launch_bounds__(1024) void k_sort_one(const int* __restrict__ ids, SortPlan p, int* key_out, int* row_out, Fill f,
                                                   int* bad_flag) {
  __shared__ unsigned item[SORT_ONE];
  __shared__ unsigned short cnt[16][DIGITS];
  __shared__ int start[DIGITS], wsum[8];
  if (clears(f)) return;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int groups = (p.n + 1023) >> 10, first = w * groups * 64 + lane;  // of 64 items, for each wave
  unsigned it[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = first + k * 64;
    it[k] = k < groups && i < p.n ? (unsigned)token_key(ids, i, p.vocab, bad_flag) << 13 | i : ~0u;
  }
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = 13 + p.shift[pass], mask = p.mask[pass];
    for (int j = t; j < 16 * DIGITS; j += 1024) (&cnt[0][0])[j] = 0;
    __syncthreads();
    int rank[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < groups) rank[k] = wave_rank(cnt[w], (it[k] >> shift) & mask, first + k * 64 < p.n);
    __syncthreads();
    int total = 0;
    if (t < DIGITS) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int c = cnt[j][t];
        cnt[j][t] = (unsigned short)total;  // of earlier waves
        total += c;
      }
    }
    const int base = digits_before(total, wsum);
    if (t < DIGITS) start[t] = base;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= groups || first + k * 64 >= p.n) continue;
      const int digit = (it[k] >> shift) & mask;
      item[start[digit] + cnt[w][digit] + rank[k]] = it[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < groups && first + k * 64 < p.n) it[k] = item[first + k * 64];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k >= groups || first + k * 64 >= p.n) continue;
    key_out[first + k * 64] = (int)(it[k] >> 13);
    row_out[first + k * 64] = (int)(it[k] & 8191);
  }
}

// Digit counts of each tile for a pass: with k_sort_scatter 4.7 + 9.3 us a pass at 131071 tokens, chains of loads that 64
// workgroups do not hide.
__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_count(const int* __restrict__ ids, SortPlan p, int pass,
                                                                const int* key_in, int* hist, Fill f, int* bad_flag) {
  __shared__ int cnt[DIGITS];
  if (clears(f)) return;
  const int t = threadIdx.x;
  if (t < DIGITS) cnt[t] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = blockIdx.x * SORT_TILE + k * (64 * SORT_WAVES) + t;
    if (i < p.n)
      atomicAdd(&cnt[((pass == 0 ? token_key(ids, i, p.vocab, bad_flag) : key_in[i]) >> p.shift[pass]) & p.mask[pass]], 1);
  }
  __syncthreads();
  if (t < DIGITS) hist[(size_t)blockIdx.x * DIGITS + t] = cnt[t];
}

// A tile's items to their places among all.  Each tile reads all tiles' counts, 2 KB x tiles^2 a pass: nothing at 64 tiles, but what a
// call of 2^22 and of 2^24 rows of 8 columns takes (1.2 and 11 ms; 2^20 0.24).
__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_scatter(const int* __restrict__ ids, SortPlan p, int pass,
                                                                  const int* __restrict__ hist, const int* key_in,
                                                                  const int* row_in, int* key_out, int* row_out, Fill f) {
  __shared__ int cnt[SORT_WAVES][DIGITS];
  __shared__ int wsum[8];
  if (clears(f)) return;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int key[4], row[4], rank[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = blockIdx.x * SORT_TILE + w * 256 + k * 64 + lane, j = min(i, p.n - 1);
    key[k] = pass == 0 ? token_key(ids, j, p.vocab, nullptr) : key_in[j];
    row[k] = pass == 0 ? j : row_in[j];
    if (i >= p.n) row[k] = -1;
  }
  // Items of this digit in all tiles, and in the tiles before this one.
  int before = 0, total = 0;
  if (t < DIGITS) {
#pragma unroll 16
    for (int j = 0; j < p.ntiles; ++j) {
      const int c = hist[(size_t)j * DIGITS + t];
      before += j < (int)blockIdx.x ? c : 0;
      total += c;
    }
#pragma unroll
    for (int j = 0; j < SORT_WAVES; ++j) cnt[j][t] = 0;
  }
  int base = digits_before(total, wsum) + before;
#pragma unroll
  for (int k = 0; k < 4; ++k) rank[k] = wave_rank(cnt[w], (key[k] >> p.shift[pass]) & p.mask[pass], row[k] >= 0);
  __syncthreads();
  if (t < DIGITS) {
#pragma unroll
    for (int j = 0; j < SORT_WAVES; ++j) {
      const int c = cnt[j][t];
      cnt[j][t] = base;
      base += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (row[k] < 0) continue;
    const int to = cnt[w][(key[k] >> p.shift[pass]) & p.mask[pass]] + rank[k];
    key_out[to] = key[k];
    row_out[to] = row[k];
  }
}

__global__ __launch_bounds__(256) void k_clear(Fill f) { clears(f); }

// ---------------------------------------------------------------- sums
// Rows are read and written through buffer descriptors: a lane behind the last column, or a row that is left out (0 columns),
// is out of range and costs no branch, which every load behind it would have to wait at.
template <int DT>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_at(const void* p, long long row, int d, bool on = true) {
  constexpr int SIZE = DT == ZO_F32 ? 4 : 2;
  return __builtin_amdgcn_make_buffer_rsrc((char*)p + (size_t)row * d * SIZE, (short)0, on ? d * SIZE : 0, 0x00020000);
}

// Eight columns of one row, as they are loaded and added.
template <int DT>
struct Row8 {
  u32x4 w[DT == ZO_F32 ? 2 : 1];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int c) {
    const int at = c * (DT == ZO_F32 ? 4 : 2);
    w[0] = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
    if constexpr (DT == ZO_F32) w[1] = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16, 0, 0);
  }
  static __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, int c, const float* v) {
    const int at = c * (DT == ZO_F32 ? 4 : 2);
    if constexpr (DT == ZO_F32) {
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, (f32x4){v[0], v[1], v[2], v[3]}), r, at, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, (f32x4){v[4], v[5], v[6], v[7]}), r, at + 16, 0, 0);
    } else if constexpr (DT == ZO_BF16) {
      __builtin_amdgcn_raw_buffer_store_b128((u32x4){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                     pack_bf16x2(v[6], v[7])}, r, at, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b128((u32x4){pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]), pack_f16x2(v[4], v[5]),
                                                     pack_f16x2(v[6], v[7])}, r, at, 0, 0);
    }
  }
  __device__ __forceinline__ void add_to(float* s) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DT == ZO_F32) {
        s[k] += __uint_as_float(w[0][k]);
        s[4 + k] += __uint_as_float(w[1][k]);
      } else if constexpr (DT == ZO_BF16) {
        s[2 * k] += __uint_as_float(w[0][k] << 16);
        s[2 * k + 1] += __uint_as_float(w[0][k] & 0xffff0000u);
      } else {
        s[2 * k] += f16_to_f32((uint16_t)w[0][k]);
        s[2 * k + 1] += f16_to_f32((uint16_t)(w[0][k] >> 16));
      }
    }
  }
};

// What a token's sum does to its row of the table's gradient; `held` is what the row holds, where it is added to.
template <int OT, bool ADD>
__device__ __forceinline__ void put_row(__amdgpu_buffer_rsrc_t r, int c, const float* s, float scale, const Row8<OT>& held) {
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if constexpr (ADD) held.add_to(v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = ADD ? fmaf(scale, s[e], v[e]) : scale * s[e];
  Row8<OT>::store(r, c, v);
}

// A few tokens need no sorting: a wave per row and 512 columns looks whether its token occurs earlier (then that row's
// wave has it), and adds up the rows where it occurs, four at a time.  Latency: ids, rows, and where it is added to the gradient's
// row; 61 rows of 4096 bf16 4.5 us.
template <int DT, int OT, bool ADD>
__global__ __launch_bounds__(256) void k_embed_few(const int* __restrict__ ids, int n, int vocab, int d,
                                                   const void* __restrict__ dH, float scale, void* dE, int* bad_flag, int nslab) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(block_of() * 4) + (threadIdx.x >> 6));
  const int t = wave / nslab, lane = threadIdx.x & 63, c = (wave - t * nslab) * 512 + lane * 8;
  if (t >= n) return;
  const int id = ids[t];
  if ((unsigned)id >= (unsigned)vocab) {
    if (id >= vocab && bad_flag && lane == 0) *bad_flag = 1;
    return;
  }
  unsigned long long where[FEW / 64];
#pragma unroll
  for (int j = 0; j < FEW / 64; ++j) where[j] = __ballot(j * 64 + lane < n && ids[min(j * 64 + lane, n - 1)] == id);
#pragma unroll
  for (int j = 0; j < FEW / 64; ++j) {
    const int upto = min(max(t - j * 64, 0), 64);
    if (where[j] & (upto == 64 ? ~0ull : (1ull << upto) - 1)) return;
  }
  const __amdgpu_buffer_rsrc_t mine = row_at<OT>(dE, id, d);
  Row8<OT> held;
  if (ADD) held.load(mine, c);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < FEW / 64; ++j) {
    unsigned long long left = where[j];
    while (left) {
      Row8<DT> r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool on = left != 0;
        r[u].load(row_at<DT>(dH, j * 64 + (on ? __builtin_ctzll(left) : 0), d, on), c);
        left &= left - 1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) r[u].add_to(s);  // a row that is left out adds zeros
    }
  }
  put_row<OT, ADD>(mine, c, s, scale, held);
}

// A wave sums 512 columns of CHUNK sorted positions, eight rows on their way at a time (four, and four of the gradient, where
// it is added to).  HBM bounds it: 131071 rows of 1024 fp32 into 151936 take 181 us, 4.5 TB/s.  Tokens that lie whole in them
// are written; the sums of one that came in from the positions before, or goes on behind, are kept: part[2 chunk] and
// part[2 chunk + 1].
template <int DT, int OT, bool ADD, int CHUNK>
__global__ __launch_bounds__(256) void k_embed_sum(const int* __restrict__ key, const int* __restrict__ row, int n, int vocab,
                                                   int d, const void* __restrict__ dH, float scale, void* dE, float* part,
                                                   int nchunk, int nslab) {
  constexpr int U = ADD ? 4 : 8;
  const long long wave = block_of() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = (int)(wave / nslab), lane = threadIdx.x & 63, c = (int)(wave - (long long)chunk * nslab) * 512 + lane * 8;
  if (chunk >= nchunk) return;
  const int i0 = chunk * CHUNK, at = i0 + lane;
  // Lane i has position i0 + i's token and row; then the token behind the last, and the one before the first.
  const int k = at < n && lane < CHUNK ? key[at] : vocab, r = at < n && lane < CHUNK ? row[at] : 0;
  const int behind = i0 + CHUNK < n ? key[i0 + CHUNK] : vocab, before = i0 > 0 ? key[i0 - 1] : -1;
  const int m = __popcll(__ballot(k < vocab));  // sorted: those that count come first
  if (m == 0) return;
  const int next = __shfl_down(k, 1, 64);
  const unsigned long long ends = __ballot(k != (lane == CHUNK - 1 ? behind : next));  // the token's last position
  bool inside = before != __builtin_amdgcn_readfirstlane(k);  // the running token began in this chunk
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < m; i += U) {
    Row8<DT> v[U];
    Row8<OT> held[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = min(i + u, m - 1);
      v[u].load(row_at<DT>(dH, __builtin_amdgcn_readlane(r, j), d, i + u < m), c);
      if (ADD) held[u].load(row_at<OT>(dE, __builtin_amdgcn_readlane(k, j), d, i + u < m && ((ends >> j) & 1)), c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= m) break;
      v[u].add_to(s);
      const bool end = (ends >> (i + u)) & 1;
      if (!end && i + u + 1 < m) continue;
      if (end && inside)
        put_row<OT, ADD>(row_at<OT>(dE, __builtin_amdgcn_readlane(k, i + u), d), c, s, scale, held[u]);
      else
        Row8<ZO_F32>::store(row_at<ZO_F32>(part, 2LL * chunk + (inside ? 1 : 0), d), c, s);
      inside = true;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 0.f;
    }
  }
}

// Joins the sums of each token that lies in more than one chunk, at the chunk where it begins, which keeps its first sum in
// part[2 chunk + 1].  A wave looks at a chunk, and 256 columns; a token of up to JOIN_ALONE further chunks it adds by itself, in
// order; longer ones the workgroup takes one after another, each wave a run of chunks, then the waves' sums in order.  The longest
// run bounds it (10 us where a token fills 9 % of 131071 rows; with 512 columns a wave, and so half as many loads on their way, 12).
template <int OT, bool ADD, int CHUNK>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_embed_join(const int* __restrict__ key, int n, int vocab, int d, float scale,
                                                                void* dE, const float* __restrict__ part, int nchunk, int nslab) {
  constexpr int U = 16;
  __shared__ f32x4 sums[JOIN_WAVES][64];
  __shared__ int reach[JOIN_WAVES];
  const long long block = block_of(), group = block / nslab;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (int)(block - group * nslab) * 256 + lane * 4, first = (int)(group * JOIN_WAVES);
  auto load = [&](long long row, bool on) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(row_at<ZO_F32>(part, row, d, on), c * 4, 0, 0));
  };
  auto add_chunks = [&](int j0, int j1, f32x4 s) {
    for (int j = j0; j < j1; j += U) {
      f32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = load(2LL * (j + u), j + u < j1);
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];  // a chunk that is left out adds zeros
    }
    return s;
  };
  auto put = [&](int chunk, f32x4 s) {
    if (c >= d) return;
    const size_t at = (size_t)key[chunk * CHUNK + CHUNK - 1] * d + c;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if constexpr (OT == ZO_F32) {
      f32x4* to = (f32x4*)((float*)dE + at);
      if (ADD) v = *to;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = ADD ? fmaf(scale, s[e], v[e]) : scale * s[e];
      *to = v;
    } else {
      u32x2* to = (u32x2*)((uint16_t*)dE + at);
      if (ADD) {
        const u32x2 h = *to;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = unpk<OT == ZO_F16>(h[e >> 1], e & 1);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = ADD ? fmaf(scale, s[e], v[e]) : scale * s[e];
      *to = (u32x2){cvt_pk<OT == ZO_F16>(v[0], v[1]), cvt_pk<OT == ZO_F16>(v[2], v[3])};
    }
  };
  const int chunk = first + w, i0 = chunk * CHUNK, last = i0 + CHUNK - 1;
  int more = 0;  // chunks behind its own that this wave's token reaches
  if (chunk < nchunk - 1) {
    const int k = key[last], behind = key[last + 1], from = key[i0], before = i0 > 0 ? key[i0 - 1] : -1;
    if (k < vocab && behind == k && !(from == k && before == k)) {
      for (bool on = true; on;) {  // 256 chunks' first tokens at a time
        int first_key[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) first_key[u] = key[min(chunk + 1 + more + u * 64 + lane, nchunk - 1) * CHUNK];
        const int base = chunk + 1 + more + lane;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const unsigned long long out = on ? ~__ballot(base + u * 64 < nchunk && first_key[u] == k) : 1ull;
          more += out ? __builtin_ctzll(out) : 64;
          on = on && out == 0;
        }
      }
    }
  }
  if (lane == 0) reach[w] = more > JOIN_ALONE ? more : 0;
  if (more > 0 && more <= JOIN_ALONE) put(chunk, add_chunks(chunk + 1, chunk + 1 + more, load(2LL * chunk + 1, true)));
  __syncthreads();
  for (int q = 0; q < JOIN_WAVES; ++q) {
    const int many = reach[q];
    if (!many) continue;
    const int each = (many + JOIN_WAVES - 1) / JOIN_WAVES, j0 = first + q + 1 + w * each, j1 = min(j0 + each, first + q + 1 + many);
    f32x4 s = add_chunks(j0, j1, load(2LL * (first + q) + 1, w == 0));
    sums[w][lane] = s;
    __syncthreads();
    if (w == 0) {
#pragma unroll
      for (int j = 1; j < JOIN_WAVES; ++j) s += sums[j][lane];
      put(first + q, s);
    }
    __syncthreads();
  }
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

namespace {
// A kernel's launch with the types of the rows and of the gradient, and whether it is added to, as constants.
template <typename F>
int embed_kernels(int dtype, int out_dtype, int accumulate, F f) {
  auto with = [&](auto dt, auto ot) { return accumulate ? f(dt, ot, std::true_type()) : f(dt, ot, std::false_type()); };
  const std::integral_constant<int, ZO_F32> f32;
  const std::integral_constant<int, ZO_BF16> bf16;
  const std::integral_constant<int, ZO_F16> f16;
  if (dtype == ZO_F32) return with(f32, f32);
  if (dtype == ZO_BF16) return out_dtype == ZO_F32 ? with(bf16, f32) : with(bf16, bf16);
  return out_dtype == ZO_F32 ? with(f16, f32) : with(f16, f16);
}
}  // namespace

int zo_embedding_launch(long long rows, int vocab, int d, int dtype, const int* ids, const void* E, float scale, void* H,
                        int* bad_flag, hipStream_t stream) {
  const int words = d / (dtype == ZO_F32 ? 4 : 8);
  const long long total = rows * words, per = 4 * 64 * SPAN;
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, grid_of((total + per - 1) / per), dim3(256), 0, stream, ids, (const u32x4*)E, scale, (u32x4*)H, bad_flag,
                       total, vocab, words);
  };
  if (dtype == ZO_F32) go(k_embedding<ZO_F32>);
  else if (dtype == ZO_BF16) go(k_embedding<ZO_BF16>);
  else go(k_embedding<ZO_F16>);
  return zo_hip_status(hipGetLastError(), "k_embedding");
}

int zo_embedding_backward_launch(long long rows, int vocab, int d, int dtype, const int* ids, const void* dH, float scale,
                                 int out_dtype, void* dE, int accumulate, int* bad_flag, void* ws, hipStream_t stream,
                                 size_t* ws_needed) {
  const SortPlan p = sort_plan(rows, vocab);
  const int n = p.n, nslab = (d + 511) / 512;
  // Positions of a wave, us with 16, 32 and 64: 4096 rows of 4096 bf16 added to fp32 36, 38, 49; 20000 121, 119, 128; 65536, dense,
  // 245, 240, 230; 100000 rows of 128 50, 46, 51.
  const int chunk = n <= 4096 ? 16 : n < 65536 || nslab == 1 ? 32 : 64, nchunk = (n + chunk - 1) / chunk;
  const bool few = n <= FEW, one = n <= SORT_ONE && vocab < (1 << 18);
  WsCarver w(ws);
  int* hist = one ? nullptr : (int*)w.take((size_t)p.ntiles * DIGITS * sizeof(int));
  int* key[2] = {(int*)w.take((size_t)n * 4), one ? nullptr : (int*)w.take((size_t)n * 4)};
  int* row[2] = {(int*)w.take((size_t)n * 4), one ? nullptr : (int*)w.take((size_t)n * 4)};
  float* part = (float*)w.take((size_t)2 * nchunk * d * sizeof(float));
  if (ws_needed) {
    *ws_needed = few ? 0 : w.off;
    return ZO_OK;
  }
  // A dense gradient is cleared first, by the sorting launches where there are some.
  const long long words = accumulate ? 0 : (long long)vocab * d / (out_dtype == ZO_F32 ? 4 : 8);
  const int launches = few || one ? 1 : 2 * p.passes;
  int at = 0;
  auto fill = [&](int sorters) {
    const Fill f = {(u32x4*)dE, words * at / launches, words * (at + 1) / launches, sorters};
    ++at;
    return f;
  };
  auto grid = [&](const Fill& f, int threads) {
    return dim3((unsigned)(f.sorters + min((f.hi - f.lo + 4 * threads - 1) / (4 * threads), 2048LL * 1024 / threads)));
  };
  int st = ZO_OK;
  if (few) {
    if (words) {
      const Fill f = fill(0);
      hipLaunchKernelGGL(k_clear, grid(f, 256), dim3(256), 0, stream, f);
      st = zo_hip_status(hipGetLastError(), "k_clear");
    }
    if (st != ZO_OK || n == 0) return st;
    return embed_kernels(dtype, out_dtype, accumulate, [&](auto dt, auto ot, auto add) {
      constexpr int DT = decltype(dt)::value, OT = decltype(ot)::value;
      constexpr bool ADD = decltype(add)::value;
      hipLaunchKernelGGL((k_embed_few<DT, OT, ADD>), grid_of(((long long)n * nslab + 3) / 4), dim3(256), 0, stream, ids, n, vocab,
                         d, dH, scale, dE, bad_flag, nslab);
      return zo_hip_status(hipGetLastError(), "k_embed_few");
    });
  }
  int last = 0;
  if (one) {
    const Fill f = fill(1);
    hipLaunchKernelGGL(k_sort_one, grid(f, 1024), dim3(1024), 0, stream, ids, p, key[0], row[0], f, bad_flag);
    st = zo_hip_status(hipGetLastError(), "k_sort_one");
  } else {
    for (int q = 0; q < p.passes && st == ZO_OK; ++q) {
      const int from = (q + 1) & 1, to = last = q & 1;
      const Fill f = fill(p.ntiles);
      hipLaunchKernelGGL(k_sort_count, grid(f, 64 * SORT_WAVES), dim3(64 * SORT_WAVES), 0, stream, ids, p, q, key[from], hist,
                         f, bad_flag);
      if ((st = zo_hip_status(hipGetLastError(), "k_sort_count")) != ZO_OK) break;
      const Fill g = fill(p.ntiles);
      hipLaunchKernelGGL(k_sort_scatter, grid(g, 64 * SORT_WAVES), dim3(64 * SORT_WAVES), 0, stream, ids, p, q, hist, key[from],
                         row[from], key[to], row[to], g);
      st = zo_hip_status(hipGetLastError(), "k_sort_scatter");
    }
  }
  if (st != ZO_OK) return st;
  const int *skey = key[last], *srow = row[last];
  return embed_kernels(dtype, out_dtype, accumulate, [&](auto dt, auto ot, auto add) {
    constexpr int DT = decltype(dt)::value, OT = decltype(ot)::value;
    constexpr bool ADD = decltype(add)::value;
    const dim3 sums = grid_of(((long long)nchunk * nslab + 3) / 4);
    const int jslab = (d + 255) / 256;
    const dim3 joins = grid_of((long long)((nchunk + JOIN_WAVES - 1) / JOIN_WAVES) * jslab);
    auto go = [&](auto sum, auto join) {
      hipLaunchKernelGGL(sum, sums, dim3(256), 0, stream, skey, srow, n, vocab, d, dH, scale, dE, part, nchunk, nslab);
      const int st = zo_hip_status(hipGetLastError(), "k_embed_sum");
      if (st != ZO_OK) return st;
      hipLaunchKernelGGL(join, joins, dim3(64 * JOIN_WAVES), 0, stream, skey, n, vocab, d, scale, dE, part, nchunk, jslab);
      return zo_hip_status(hipGetLastError(), "k_embed_join");
    };
    return chunk == 16   ? go(k_embed_sum<DT, OT, ADD, 16>, k_embed_join<OT, ADD, 16>)
           : chunk == 32 ? go(k_embed_sum<DT, OT, ADD, 32>, k_embed_join<OT, ADD, 32>)
                         : go(k_embed_sum<DT, OT, ADD, 64>, k_embed_join<OT, ADD, 64>);
  });
}
