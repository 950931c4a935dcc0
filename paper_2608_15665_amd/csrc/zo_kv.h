// Device side of a paged key/value batch (KvArgs): a sequence's rows and lengths, its pages.  Every
// number read from device memory is checked here before it becomes an address.
#pragma once

#include "zo_internal.h"

namespace {

// The grid of a launch of n < 2^31 workgroups of 256 threads: the x dimension holds fewer than 2^32 threads, so from 2^24
// workgroups on they go in rows of 2^22, of which the last may be longer than n.
inline dim3 kv_grid(long long n) {
  if (n < (1LL << 24)) return dim3((unsigned)n);
  return dim3(1u << 22, (unsigned)((n + (1LL << 22) - 1) >> 22));
}
__device__ __forceinline__ unsigned kv_block() { return blockIdx.x + (blockIdx.y << 22); }

// A sequence's first row, its rows and its length with them.
struct KvSpan {
  int r0, n, len;
};

__host__ __device__ __forceinline__ KvSpan kv_span(const KvArgs& a, int s) {
  KvSpan sp;
  // A length below -2^30 is as much padding as that one, and its first position does not wrap.
  sp.len = max(a.kv_len[s], -(1 << 30));
  if (!a.q_start) {
    sp.r0 = s;
    sp.n = 1;
    return sp;
  }
  const int q0 = a.q_start[s], q1 = a.q_start[s + 1];
  sp.r0 = min(max(q0, 0), a.rows);
  sp.n = min(max(q1, sp.r0), a.rows) - sp.r0;
  if (a.bad_flag && (sp.r0 != q0 || sp.r0 + sp.n != q1 || sp.n > a.max_q)) *a.bad_flag = 1;
  return sp;
}

// Positions that the table has.
__host__ __device__ __forceinline__ int kv_cap(const KvArgs& a) { return a.max_pages << a.log2ps; }

// Page j of sequence s, or -1 where the table has none or a bad one.
__host__ __device__ __forceinline__ int kv_page(const KvArgs& a, int s, int j) {
  if (j >= a.max_pages) return -1;
  const int page = a.table[(size_t)s * a.max_pages + j];
  return (unsigned)page < (unsigned)a.num_pages ? page : -1;
}

}  // namespace
