// Appending to a paged key/value cache, keys and queries rotated to their positions on the way:
// what a layer of the LLaMA family does between its q, k, v products and its attention when it
// answers token by token (the rotation of zo_rope, at positions that are not 0, 1, ...).
//
// A row's angles are the same for all its heads: a team of waves forms the dh / 2 sines and cosines
// of a row once, in LDS, and then turns every head of Q and K and copies V with 16-byte accesses.
#include "zo_attn.h"
#include "zo_kv.h"

namespace {

struct AppendArgs {
  KvArgs kv;
  const void *Q, *K, *V;
  void* Qo;
  long long ldq, ldqo, ldk, ldv;
  double k;    // log2 of the frequency of dimension 1: -2 log2(base) / dh; 0: no rotation
  int tiles;   // workgroups along a sequence (16-bit), pages of a sequence (8-bit)
  int parts;   // workgroups per row (16-bit), head groups (8-bit)
  int qblocks; // 8-bit: workgroups that rotate Q, before those of the pages
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

// Fills t[i] = (cos, sin) of row position p, i = first, first + step, ... < half.
__device__ __forceinline__ void fill_turns(float2* t, int half, int first, int step, int p, double k) {
  for (int i = first; i < half; i += step) {
    float sn, cs;
    turn((double)p * (exp2((double)i * k) * kInv2Pi), sn, cs);
    t[i] = make_float2(cs, sn);
  }
}

// Row `row` of the call: items y = 0 .. heads dh / 16 - 1 turn Q, the next kv_heads dh / 16 turn K,
// the rest copy V (without a rotation: K, then V) into slot `slot` of the cache, in elements of
// head 0's page (-1: not stored).
template <int DT, int WPT>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int s, int tile, int part, float2 (*turns)[64]) {
  const int dh = a.kv.dh, half = dh / 2, TB = 4 / WPT;
  const KvSpan sp = kv_span(a.kv, s);
  const int nq = min(sp.n, a.kv.max_q);
  if (tile * TB >= nq) return;
  const int team = threadIdx.x / (64 * WPT), tl = threadIdx.x % (64 * WPT);
  const int i = tile * TB + team;
  const bool mine = i < nq;
  const int p = sp.len - sp.n + i, pr = max(p, 0);
  if (a.k != 0.0 && mine) fill_turns(turns[team], half, tl, 64 * WPT, pr, a.k);
  long long slot = -1;  // element of head 0 in the cache
  if (mine && p >= 0 && a.kv.K) {
    const int page = kv_page(a.kv, s, p >> a.kv.log2ps);
    if (page >= 0) slot = ((((long long)page * a.kv.kv_heads) << a.kv.log2ps) + (p & ((1 << a.kv.log2ps) - 1))) * dh;
    else if (a.kv.bad_flag) *a.kv.bad_flag = 1;
  }
  __syncthreads();
  if (!mine) return;
  const long long row = sp.r0 + i;
  const bool rot = a.k != 0.0;
  const int cph = dh / 16;  // rotated chunks (8 pairs) per head
  const int nq_items = rot && a.Q ? a.kv.heads * cph : 0, nk = a.kv.K ? a.kv.kv_heads * cph : 0;
  const int n_rot = nq_items + (rot ? nk : 0), n_all = n_rot + (rot ? 2 * nk : 4 * nk);
  const int lcph = dh == 128 ? 3 : 2;
  const long long hstride = (long long)dh << a.kv.log2ps;
  for (int y = part * 64 * WPT + tl; y < n_all; y += a.parts * 64 * WPT) {
    if (y < n_rot) {
      const bool isq = y < nq_items;
      const int x = isq ? y : y - nq_items;
      const int h = x >> lcph, c = x & (cph - 1);
      const size_t src = (isq ? row * a.ldq : row * a.ldk) + (size_t)h * dh + 8 * c;
      float u[8], v[8];
      load8<DT>(isq ? a.Q : a.K, src, u);
      load8<DT>(isq ? a.Q : a.K, src + half, v);
      rotate8(u, v, &turns[team][8 * c]);
      if (!isq && slot < 0) continue;
      const size_t dst = isq ? (size_t)(row * a.ldqo) + (size_t)h * dh + 8 * c : (size_t)(slot + h * hstride) + 8 * c;
      store8<DT>(isq ? a.Qo : a.kv.K, dst, u);
      store8<DT>(isq ? a.Qo : a.kv.K, dst + half, v);
    } else if (slot >= 0) {
      const int x = y - n_rot;
      const bool isk = !rot && x < 2 * nk;
      const int z = !rot && !isk ? x - 2 * nk : x;
      const int h = z >> (lcph + 1), c = z & (2 * cph - 1);
      const uint16_t* src = (const uint16_t*)(isk ? a.K : a.V) + (isk ? row * a.ldk : row * a.ldv) + (size_t)h * dh + 8 * c;
      *(u32x4*)((uint16_t*)(isk ? a.kv.K : a.kv.V) + (size_t)(slot + h * hstride) + 8 * c) = *(const u32x4*)src;
    }
  }
}

template <int DT, int WPT>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  __shared__ float2 turns[4][64];
  const int w = blockIdx.x, part = w % a.parts, t = w / a.parts;
  append_rows<DT, WPT>(a, t / a.tiles, t % a.tiles, part, turns);
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
__device__ __forceinline__ u32x2 codes8(const float* v, float inv) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fabsf(v[e]) < INFINITY ? v[e] * inv : __builtin_nanf("");
  return (u32x2){codes4(x), codes4(x + 4)};
}

// One page of one sequence, for the head group `part`: wave w takes tensor w & 1 (K, V) of heads
// w >> 1, w >> 1 + 2, ... of the group.  Two passes over the page's new rows (the largest magnitude,
// then the codes; the second reads them from the caches), and one over its earlier slots where the
// scale grows.
template <int DT>
__device__ __forceinline__ void append_page8(const AppendArgs& a, int s, int jpage, int part, float2 (*turns)[64]) {
  const KvArgs& kv = a.kv;
  const int dh = kv.dh, half = dh / 2, ps = 1 << kv.log2ps, cph = dh / 16;
  const KvSpan sp = kv_span(kv, s);
  const int p0 = sp.len - sp.n;                                // position of the sequence's row 0
  const int pend = min(p0 + min(sp.n, kv.max_q), kv_cap(kv));  // positions stored end here
  const int pbeg = max(p0, 0);
  const int j = (pbeg >> kv.log2ps) + jpage;
  const int lo = max(pbeg, j << kv.log2ps), hi = min(pend, (j + 1) << kv.log2ps);
  if (jpage == 0 && part == 0 && threadIdx.x == 0 && kv.bad_flag && p0 + min(sp.n, kv.max_q) > kv_cap(kv)) *kv.bad_flag = 1;
  if (lo >= hi) return;
  const int page = kv_page(kv, s, j);
  if (page < 0) {
    if (kv.bad_flag && threadIdx.x == 0) *kv.bad_flag = 1;
    return;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int nt = hi - lo, old = lo & (ps - 1);
  const int hper = (kv.kv_heads + a.parts - 1) / a.parts;
  const int h0 = part * hper, h1 = min(h0 + hper, kv.kv_heads);
  const int lcph = dh == 128 ? 3 : 2;
  const bool rot = a.k != 0.0;
  const bool isk = (wave & 1) == 0;
  const double theta = rot ? exp2((double)(threadIdx.x & (half - 1)) * a.k) * kInv2Pi : 0.0;
  const long long row0 = sp.r0 + (lo - p0);
  const uint16_t* src = (const uint16_t*)(isk ? a.K : a.V);
  const long long ld = isk ? a.ldk : a.ldv;
  // Heads in steps of 2; the rows in chunks of 64, whose turns fit LDS.  All waves take the same
  // steps, so that they meet at the barriers.
  for (int hb = h0; hb < h1; hb += 2) {
    const int h = hb + (wave >> 1);
    const bool mine = h < h1;
    float amax = 0.f, inv = 0.f;
    uint8_t* base = (uint8_t*)(isk ? kv.K : kv.V) + ((((size_t)page * kv.kv_heads + (mine ? h : 0)) << kv.log2ps) * dh);
    for (int pass = 0; pass < 2; ++pass) {
      for (int c0 = 0; c0 < nt; c0 += 64) {
        const int cn = min(64, nt - c0);
        if (rot && (nt > 64 || (hb == h0 && pass == 0))) {
          __syncthreads();  // the chunk before has been used
          for (int t = threadIdx.x / half; t < cn; t += 256 / half) {
            float sn, cs;
            turn((double)(lo + c0 + t) * theta, sn, cs);
            turns[t][threadIdx.x & (half - 1)] = make_float2(cs, sn);
          }
          __syncthreads();
        }
        if (!mine) continue;
        for (int x = lane; x < cn * cph; x += 64) {
          const int t = x >> lcph, c = x & (cph - 1);
          const size_t at = (size_t)((row0 + c0 + t) * ld) + (size_t)h * dh + 8 * c;
          float u[8], v[8];
          load8<DT>(src, at, u);
          load8<DT>(src, at + half, v);
          if (rot && isk) rotate8(u, v, &turns[t][8 * c]);
          if (pass == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fmaxf(finite_abs(u[e]), finite_abs(v[e])));
          } else {
            uint8_t* dst = base + (size_t)(old + c0 + t) * dh + 8 * c;
            *(u32x2*)dst = codes8(u, inv);
            *(u32x2*)(dst + half) = codes8(v, inv);
          }
        }
      }
      if (pass == 0 && mine) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
        float* sc = (isk ? kv.ks : kv.vs) + (size_t)page * kv.kv_heads + h;
        float to = need_scale(amax);
        if (old > 0) {
          const float was = *sc;
          to = fmaxf(was, to);
          if (to > was) {
            const float ratio = was / to;
            for (int x = lane; x < old * dh / 8; x += 64) {
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
        if (lane == 0) *sc = to;
        inv = 1.f / to;
      }
    }
  }
}

template <int DT>
__global__ __launch_bounds__(256) void k_kv_append8(AppendArgs a, AppendArgs q) {
  __shared__ float2 turns[64][64];
  const int w = blockIdx.x;
  if (w < a.qblocks) {
    const int part = w % q.parts, t = w / q.parts;
    append_rows<DT, 1>(q, t / q.tiles, t % q.tiles, part, turns);
  } else {
    const int v = w - a.qblocks, part = v % a.parts, t = v / a.parts;
    append_page8<DT>(a, t / a.tiles, t % a.tiles, part, turns);
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
  a.qblocks = 0;
  const int cph = kv.dh / 16;
  const bool rot = a.k != 0.0;
  long long wg = 0;
  if (!kv.e8) {
    const int items = (rot && Q ? kv.heads * cph : 0) + kv.kv_heads * cph * (rot ? 3 : 4);
    // Few rows: one row per workgroup, an item per thread; many: one row per wave.
    const bool few = (long long)kv.nseq * kv.max_q <= 1024;
    a.tiles = few ? kv.max_q : (kv.max_q + 3) / 4;
    a.parts = few ? (items + 255) / 256 : 1;
    wg = (long long)kv.nseq * a.tiles * a.parts;
    if (wg <= 0x7fffffffLL) {
      const dim3 grid((unsigned)wg), block(256);
      if (few) {
        if (kv.dtype == ZO_BF16) hipLaunchKernelGGL((k_kv_append<ZO_BF16, 4>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_kv_append<ZO_F16, 4>), grid, block, 0, stream, a);
      } else {
        if (kv.dtype == ZO_BF16) hipLaunchKernelGGL((k_kv_append<ZO_BF16, 1>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_kv_append<ZO_F16, 1>), grid, block, 0, stream, a);
      }
      return zo_hip_status(hipGetLastError(), "k_kv_append");
    }
  } else {
    AppendArgs q = a;  // the queries' part: nothing is stored in the cache
    q.kv.K = nullptr;
    q.tiles = (kv.max_q + 3) / 4;
    q.parts = 1;
    const long long qb = Q ? (long long)kv.nseq * q.tiles : 0;
    a.tiles = ((kv.max_q - 1 + (1 << kv.log2ps) - 1) >> kv.log2ps) + 1;  // pages that max_q positions touch at most
    a.parts = (kv.kv_heads + 1) / 2;
    wg = qb + (long long)kv.nseq * a.tiles * a.parts;
    if (wg <= 0x7fffffffLL) {
      a.qblocks = (int)qb;
      const dim3 grid((unsigned)wg), block(256);
      if (kv.dtype == ZO_BF16) hipLaunchKernelGGL(k_kv_append8<ZO_BF16>, grid, block, 0, stream, a, q);
      else hipLaunchKernelGGL(k_kv_append8<ZO_F16>, grid, block, 0, stream, a, q);
      return zo_hip_status(hipGetLastError(), "k_kv_append8");
    }
  }
  zo_set_error("kv_append: too many workgroups (%lld)", wg);
  return ZO_ERR_UNSUPPORTED;
}
