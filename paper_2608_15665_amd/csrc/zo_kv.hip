// Appending to a paged key/value cache, keys and queries rotated to their positions on the way:
// what a layer of the LLaMA family does between its q, k, v products and its attention when it
// answers token by token (the rotation of zo_rope, at positions that are not 0, 1, ...).
//
// Bound by the bytes of Q, K and V in and out, or by the latency of a few dependent loads (a length, a page, the
// row).  A row's angles are the same for all its heads, so a workgroup takes (a part of) one row: 256 items of
// 16 bytes copied or 32 turned, one per thread, loaded before its first waves form the row's dh / 2 sines and
// cosines in LDS.  16 prompts of up to 512 rows, 40 query and 8 key heads of 128: 33 us for 145 MB where the tensors
// change from call to call (4.4 TB/s), 27 over the same ones again.  One row per wave instead, eight items after one
// another, took 37 us where this took 29, and a workgroup per whole row 38.
// A token alone is a launch's latency (3.3 us of the GPU, 61 tokens 3.9).
// The 8-bit form: one wave or two take one page of one head and tensor, for which they need the largest magnitude first
// (61 tokens 5.4 us, 16 prompts of up to 512 rows, 32 heads of 64 unrotated, 17.5 us: 3.6 TB/s).
#include "zo_attn.h"
#include "zo_kv.h"

namespace {

struct AppendArgs {
  KvArgs kv;
  const void *Q, *K, *V;
  void* Qo;
  long long ldq, ldqo, ldk, ldv;
  double k;     // log2 of the frequency of dimension 1: -2 log2(base) / dh; 0: no rotation
  int parts;    // workgroups per row
  int pages, groups;  // 8-bit: pages that max_q positions touch at most, workgroups (pairs of heads) per page
  int qblocks;  // 8-bit: workgroups that rotate Q, before those of the pages
  unsigned wgs;  // workgroups of the launch
};

// Sine and cosine of `turns` full turns: the nearest quarter turn is taken off in fp64, the rest
// (at most pi / 4) enters the Taylor polynomials, whose next terms are below 2^-29.
__device__ __forceinline__ void turn(double turns, float& sn, float& cs) {
  const double qd = rint(turns * 4.0);
  const float y = (float)(fma(qd, -0.25, turns) * 6.283185307179586);
  const float z = y * y;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(z, s, 8.3333333e-3f);
  s = fmaf(z, s, -1.6666667e-1f);
  s = fmaf(z * y, s, y);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(z, c, -1.3888889e-3f);
  c = fmaf(z, c, 4.1666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const int q = (int)fma(rint(qd * 0.25), -4.0, qd);  // -2 .. 2
  const float a = (q & 1) ? c : s, b = (q & 1) ? s : c;
  sn = (q & 2) ? -a : a;
  cs = ((q + 1) & 2) ? -b : b;
}

constexpr double kInv2Pi = 0.15915494309189535;

// The rotation of 8 pairs, its products and sums each rounded to fp32.
__device__ __forceinline__ void rotate8(float* a, float* b, const float2* cs) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = a[e] * cs[e].x - b[e] * cs[e].y, y = b[e] * cs[e].x + a[e] * cs[e].y;
    a[e] = x;
    b[e] = y;
  }
}

// Eight 16-bit values widened.
template <int DT>
__device__ __forceinline__ void widen(u32x4 w, float* v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = unpk<DT == ZO_F16>(w[e], 0);
    v[2 * e + 1] = unpk<DT == ZO_F16>(w[e], 1);
  }
}

// New row i of sequence s, items 256 part .. + 255: the first heads dh / 16 turn Q, the next kv_heads dh / 16 turn
// K, the rest copy V (without a rotation: K, then V) into the row's slot of the cache.  KV: else Q alone.
template <int DT, bool KV>
__device__ __forceinline__ void append_row(const AppendArgs& a, int s, int i, int part, float2* turns) {
  const int dh = a.kv.dh, half = dh / 2;
  const KvSpan sp = kv_span(a.kv, s);
  if (i >= min(sp.n, a.kv.max_q)) return;
  const int p = sp.len - sp.n + i;
  const long long row = sp.r0 + i;
  const bool rot = a.k != 0.0;
  const int cph = dh / 16, lcph = dh == 128 ? 3 : 2;  // rotated chunks (8 pairs) per head
  const int nq = rot && a.Q ? a.kv.heads * cph : 0, nk = KV ? a.kv.kv_heads * cph : 0;
  const int n_rot = nq + (rot ? nk : 0), n_all = n_rot + (rot ? 2 * nk : 4 * nk);
  const int y = part * 256 + threadIdx.x;
  // What this thread turns (isq: of Q, else of K) or copies (isk: K, else V): item x of it.
  const bool turned = y < n_rot, isq = y < nq, isk = turned || (!rot && y < 2 * nk);
  const int x = turned ? (isq ? y : y - nq) : y - n_rot - (rot || isk ? 0 : 2 * nk);
  const uint16_t* src = (const uint16_t*)(isq ? a.Q : isk ? a.K : a.V) + row * (isq ? a.ldq : isk ? a.ldk : a.ldv);
  u32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (turned) {
    src += (x >> lcph) * dh + 8 * (x & (cph - 1));
    u = *(const u32x4*)src;
    v = *(const u32x4*)(src + half);
  } else if (y < n_all) {
    u = *(const u32x4*)(src + 8 * x);
  }
  if (rot) {
    if ((int)threadIdx.x < half) {
      float sn, cs;
      turn((double)max(p, 0) * (exp2((double)threadIdx.x * a.k) * kInv2Pi), sn, cs);
      turns[threadIdx.x] = make_float2(cs, sn);
    }
  }
  long long slot = -1;  // element of head 0 in the cache; -1: the row is not stored
  if (KV && p >= 0) {
    const int page = kv_page(a.kv, s, p >> a.kv.log2ps);
    if (page >= 0) slot = ((((long long)page * a.kv.kv_heads) << a.kv.log2ps) + (p & ((1 << a.kv.log2ps) - 1))) * dh;
    else if (a.kv.bad_flag) *a.kv.bad_flag = 1;
  }
  if (rot) __syncthreads();
  const long long hstride = (long long)dh << a.kv.log2ps;
  if (turned) {
    const int h = x >> lcph, c = x & (cph - 1);
    if (!isq && slot < 0) return;
    if (p < 0) {  // padding: its queries are copied
      uint16_t* dst = (uint16_t*)a.Qo + row * a.ldqo + h * dh + 8 * c;
      *(u32x4*)dst = u;
      *(u32x4*)(dst + half) = v;
      return;
    }
    float f[8], g[8];
    widen<DT>(u, f);
    widen<DT>(v, g);
    rotate8(f, g, &turns[8 * c]);
    const size_t dst = isq ? (size_t)(row * a.ldqo) + (size_t)h * dh + 8 * c : (size_t)(slot + h * hstride) + 8 * c;
    store8<DT>(isq ? a.Qo : a.kv.K, dst, f);
    store8<DT>(isq ? a.Qo : a.kv.K, dst + half, g);
  } else if (y < n_all && slot >= 0) {
    const int h = x >> (lcph + 1), c = x & (2 * cph - 1);
    *(u32x4*)((uint16_t*)(isk ? a.kv.K : a.kv.V) + (size_t)(slot + h * hstride) + 8 * c) = u;
  }
}

template <int DT, bool KV>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  __shared__ float2 turns[64];
  if (kv_block() >= a.wgs) return;
  const int w = kv_block(), part = w % a.parts, t = w / a.parts;
  append_row<DT, KV>(a, t / a.kv.max_q, t % a.kv.max_q, part, turns);
}

// ---------------------------------------------------------------- 8-bit cache
__device__ __forceinline__ float finite_abs(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.f;
}

// The smallest power of two s with amax <= 448 s (448 = 1.75 2^8), within [2^-126, 2^120]: from the
// exponent and significand of amax, exactly.
__device__ __forceinline__ float need_scale(float amax) {
  int e = 0;
  const float m = frexpf(amax, &e);  // amax = m 2^e, m in [0.5, 1); 0 = 0 2^0
  e = amax > 0.f ? min(max(e - 9 + (m > 0.875f ? 1 : 0), -126), 120) : -126;
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Four codes of values already divided by the scale, to nearest even; not finite: NaN.
__device__ __forceinline__ uint32_t codes4(const float* v) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
  return (uint32_t)w;
}
// inv = 1 / to: v inv is v / to where to is a power of two, as all scales are that this file forms; with another one's
// scale it is made so by what is left of v.
__device__ __forceinline__ u32x2 codes8(const float* v, float to, float inv) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = v[e] * inv;
    x[e] = fabsf(v[e]) < INFINITY ? fmaf(fmaf(-q, to, v[e]), inv, q) : __builtin_nanf("");
  }
  return (u32x2){codes4(x), codes4(x + 4)};
}

// One page of one sequence, W waves for one head's K or V: wave w takes tensor w & 1 (K, V) of head 2 part + (w >> 1) or,
// with W = 2, of head part, each wave every other item.  Two passes
// over the page's new rows, the largest magnitude and then the codes (the second reads the rows from the caches: held
// in registers, they left room for half as many waves, and 16 prompts of 512 rows, 8 key heads of 128 and 40
// query heads, took 94 us where this took 57), and one over its earlier slots where the scale grows.
template <int DT, int DH, bool ROT, int W>
__device__ __forceinline__ void append_page8(const AppendArgs& a, int s, int jpage, int part, float2 (*turns)[64],
                                             float* tops) {
  const KvArgs& kv = a.kv;
  constexpr int half = DH / 2, CPH = DH / 16, UN = 2;  // chunks of 8 pairs of a row; items of a lane loaded together
  const int ps = 1 << kv.log2ps;
  const KvSpan sp = kv_span(kv, s);
  const int p0 = sp.len - sp.n;  // position of the sequence's row 0
  const int plast = p0 + min(sp.n, kv.max_q), pend = min(plast, kv_cap(kv));  // positions stored end at pend
  const int pbeg = max(p0, 0);
  const int j = (pbeg >> kv.log2ps) + jpage;
  const int lo = max(pbeg, j << kv.log2ps), hi = min(pend, (j + 1) << kv.log2ps);
  if (jpage == 0 && part == 0 && threadIdx.x == 0 && kv.bad_flag && plast > kv_cap(kv)) *kv.bad_flag = 1;
  if (lo >= hi) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int nt = hi - lo, old = lo & (ps - 1);
  const int h = W == 1 ? 2 * part + (wave >> 1) : part, of = W == 1 ? 0 : wave >> 1;  // of: which of the W
  const bool isk = (wave & 1) == 0, mine = h < kv.kv_heads;
  const uint16_t* src = (const uint16_t*)(isk ? a.K : a.V) + (size_t)h * DH;
  const long long ld = isk ? a.ldk : a.ldv, row0 = sp.r0 + (lo - p0);
  const int page = kv_page(kv, s, j);
  if (page < 0) {  // of all waves
    if (kv.bad_flag && threadIdx.x == 0) *kv.bad_flag = 1;
    return;
  }
  const size_t head = (size_t)page * kv.kv_heads + (mine ? h : 0);
  float* const sc = (isk ? kv.ks : kv.vs) + head;
  uint8_t* const base = (uint8_t*)(isk ? kv.K : kv.V) + ((head << kv.log2ps) * DH);
  const float was = old > 0 ? *sc : 0.f;
  const double theta = ROT ? exp2((double)(threadIdx.x & (half - 1)) * a.k) * kInv2Pi : 0.0;
  float amax = 0.f, to = 0.f, inv = 0.f;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    // 64 rows at a time: their turns fit LDS (and serve both passes where they are all).
    for (int c0 = 0; c0 < nt; c0 += 64) {
      const int cn = min(64, nt - c0), items = mine ? cn * CPH : 0;
      u32x4 u[UN], v[UN];
      auto load = [&](int x0) {  // item x: chunk x % CPH of row x / CPH
#pragma unroll
        for (int q = 0; q < UN; ++q)
          if (x0 + 64 * q < items) {
            const uint16_t* p = src + (row0 + c0 + (x0 + 64 * q) / CPH) * ld + 8 * ((x0 + 64 * q) % CPH);
            u[q] = *(const u32x4*)p;
            v[q] = *(const u32x4*)(p + half);
          }
      };
      const int first = lane + 64 * UN * of;
      load(first);
      if (ROT && (nt > 64 || pass == 0)) {
        __syncthreads();  // those before have been used
        for (int t = threadIdx.x / half; t < cn; t += 256 / half) {
          float sn, cs;
          turn((double)(lo + c0 + t) * theta, sn, cs);
          turns[t][threadIdx.x & (half - 1)] = make_float2(cs, sn);
        }
        __syncthreads();
      }
      for (int x0 = first; x0 < items; x0 += 64 * UN * W) {
#pragma unroll
        for (int q = 0; q < UN; ++q) {
          const int x = x0 + 64 * q;
          if (x < items) {
            float f[8], g[8];
            widen<DT>(u[q], f);
            widen<DT>(v[q], g);
            if (ROT && isk) rotate8(f, g, &turns[x / CPH][8 * (x % CPH)]);
            if (pass == 0) {
#pragma unroll
              for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fmaxf(finite_abs(f[e]), finite_abs(g[e])));
            } else {
              uint8_t* dst = base + (size_t)(old + c0 + x / CPH) * DH + 8 * (x % CPH);
              *(u32x2*)dst = codes8(f, to, inv);
              *(u32x2*)(dst + half) = codes8(g, to, inv);
            }
          }
        }
        load(x0 + 64 * UN * W);
      }
    }
    if (pass == 0 && mine) {
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
      if constexpr (W == 2) {  // mine is true of all waves
        if (lane == 0) tops[wave] = amax;
        __syncthreads();
        amax = fmaxf(amax, tops[wave ^ 2]);
      }
      to = need_scale(amax);
      if (old > 0) {
        to = fmaxf(was, to);
        if (to > was) {
          const float ratio = was / to;
          for (int x = lane + 64 * of; x < old * DH / 8; x += 64 * W) {
            const u32x2 w = *(const u32x2*)(base + 8 * x);
            float v[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              v[4 * e] = __builtin_amdgcn_cvt_f32_fp8(w[e], 0) * ratio;
              v[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8(w[e], 1) * ratio;
              v[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8(w[e], 2) * ratio;
              v[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8(w[e], 3) * ratio;
            }
            *(u32x2*)(base + 8 * x) = (u32x2){codes4(v), codes4(v + 4)};
          }
        }
      }
      if (lane == 0 && of == 0) *sc = to;
      inv = 1.f / to;
    }
  }
}

template <int DT, int DH, bool ROT, int W>
__global__ __launch_bounds__(256, ROT ? 4 : 5) void k_kv_append8(AppendArgs a) {
  __shared__ float2 turns[ROT ? 64 : 1][64];
  __shared__ float tops[4];
  if (kv_block() >= a.wgs) return;
  const int w = kv_block();
  if (w < a.qblocks) {
    const int part = w % a.parts, t = w / a.parts;
    append_row<DT, false>(a, t / a.kv.max_q, t % a.kv.max_q, part, turns[0]);
  } else {
    const int v = w - a.qblocks, part = v % a.groups, t = v / a.groups;
    append_page8<DT, DH, ROT, W>(a, t / a.pages, t % a.pages, part, turns, tops);
  }
}

}  // namespace

int zo_kv_append_launch(const KvArgs& kv, const void* Q, long long ldq, void* Q_out, long long ldqo, const void* K,
                        long long ldk, const void* V, long long ldv, float rope_base, hipStream_t stream) {
  AppendArgs a;
  a.kv = kv;
  a.Q = Q;
  a.Qo = Q_out;
  a.K = K;
  a.V = V;
  a.ldq = ldq;
  a.ldqo = ldqo;
  a.ldk = ldk;
  a.ldv = ldv;
  a.k = rope_base > 0.f ? -2.0 * log2((double)rope_base) / (double)kv.dh : 0.0;
  const bool rot = a.k != 0.0;
  const long long rows = (long long)kv.nseq * kv.max_q;
  if (rows > 0x7fffffffLL) {  // what follows of it stays within 64 bits
    zo_set_error("kv_append: nseq x max_q = %lld too many", rows);
    return ZO_ERR_UNSUPPORTED;
  }
  const int items = (Q ? kv.heads * (kv.dh / 16) : 0) + (kv.e8 ? 0 : kv.kv_heads * (kv.dh / 16) * (rot ? 3 : 4));
  a.parts = (items + 255) / 256;
  a.pages = a.groups = a.qblocks = 0;
  long long wg = rows * a.parts;
  const dim3 block(256);
  int st = ZO_OK;
  if (kv.e8) {
    // Q's rows in the pages' launch, or, where they are many, in one of their own: its workgroups need half of the
    // registers and no tables of turns (the prompts above, 64 positions, 40 query heads: 52 us, in one launch 55).
    const bool apart = rows > 1024;
    const long long qb = apart ? 0 : wg;
    a.pages = ((kv.max_q - 1 + (1 << kv.log2ps) - 1) >> kv.log2ps) + 1;
    // Two waves a page, head and tensor where a page of 64 positions or more may get more rows than one wave loads at
    // once (128 pairs of 8 values): there is more to such a page, and there are fewer of them.  16 prompts of 512 rows, 8 key
    // heads of 128, without and (in brackets) with 40 rotated query heads, us with two waves and with one: 256 positions
    // 26 and 36 (73, 84), 128 positions 20 and 24 (61, 65), 64 positions 17 and 19 (49, 52), 32 positions 17.3 and 16.8
    // (50, 48), 16 positions 22 and 17 (58, 49).  Single tokens of 61 sequences 5.0 and 4.6 (5.7, 5.2), of 200 7.7 and 6.3
    // (9.8, 7.6), of one 4.2 and 4.7 (4.7, 5.2), with pages of any size, in a graph.
    const bool two = kv.log2ps >= 6 && (long long)kv.max_q * (kv.dh / 16) > 128;
    a.groups = two ? kv.kv_heads : (kv.kv_heads + 1) / 2;
    const long long pages = qb + (long long)kv.nseq * a.pages * a.groups;
    if (pages > 0x7fffffffLL || wg > 0x7fffffffLL) {
      zo_set_error("kv_append: too many workgroups (%lld)", pages + wg);
      return ZO_ERR_UNSUPPORTED;
    }
    a.qblocks = (int)qb;
    const dim3 grid = kv_grid(pages);
    a.wgs = (unsigned)pages;
#define ZO_APPEND8_W(T, D, R)                                                                        \
  if (two) hipLaunchKernelGGL((k_kv_append8<T, D, R, 2>), grid, block, 0, stream, a);                \
  else hipLaunchKernelGGL((k_kv_append8<T, D, R, 1>), grid, block, 0, stream, a)
#define ZO_APPEND8(D, R)                                                                             \
  if (kv.dtype == ZO_BF16) { ZO_APPEND8_W(ZO_BF16, D, R); } else { ZO_APPEND8_W(ZO_F16, D, R); }
    if (kv.dh == 64) {
      if (rot) { ZO_APPEND8(64, true); } else { ZO_APPEND8(64, false); }
    } else {
      if (rot) { ZO_APPEND8(128, true); } else { ZO_APPEND8(128, false); }
    }
#undef ZO_APPEND8
#undef ZO_APPEND8_W
    st = zo_hip_status(hipGetLastError(), "k_kv_append8");
    if (st != ZO_OK || !apart || wg == 0) return st;
    a.wgs = (unsigned)wg;
    if (kv.dtype == ZO_BF16) hipLaunchKernelGGL((k_kv_append<ZO_BF16, false>), kv_grid(wg), block, 0, stream, a);
    else hipLaunchKernelGGL((k_kv_append<ZO_F16, false>), kv_grid(wg), block, 0, stream, a);
    return zo_hip_status(hipGetLastError(), "k_kv_append");
  }
  if (wg <= 0x7fffffffLL) {
    a.wgs = (unsigned)wg;
    if (kv.dtype == ZO_BF16) hipLaunchKernelGGL((k_kv_append<ZO_BF16, true>), kv_grid(wg), block, 0, stream, a);
    else hipLaunchKernelGGL((k_kv_append<ZO_F16, true>), kv_grid(wg), block, 0, stream, a);
    return zo_hip_status(hipGetLastError(), "k_kv_append");
  }
  zo_set_error("kv_append: too many workgroups (%lld)", wg);
  return ZO_ERR_UNSUPPORTED;
}
