// Causal attention over a paged key/value cache: few queries (a token, some drafted tokens, a piece
// of a prompt) against many keys.
//
// The queries of the heads that share a key/value head read the same keys, so a workgroup's rows are
// (token, head of the group) pairs of one key/value head: row t G + j is head j of the group at the
// sequence's new token t.
//
// k_paged_rows: a workgroup of 4 waves takes 16 NG rows and a range of the keys; its waves take the
// range's tiles of 32 keys in turn, each with a softmax of its own (running maximum and sum), and
// join their results in LDS at the end.  Ranges of one sequence (nsplit > 1) are joined by
// k_paged_join.  Products as in the causal attention of whole sequences:
//   S^T = K Q^T   (16 x 16 x 32 MFMA; A = K rows from global memory straight into the fragment)
//   O^T += V^T P^T, V^T's fragments by transposed reads of a row-major V tile in LDS, private to
//   the wave; P as a hi + lo 16-bit pair.
// 8-bit caches: codes are exact in fp16 and in bf16, so K enters as Q's type, V as bf16; the page's
// key scale multiplies S, its value scale P, in fp32.
// A page boundary never lies inside 16 keys, so the 16 keys of an MFMA tile have one page: its
// number is uniform over the wave.  Page numbers are read 64 at a time, one per lane.
#include "zo_attn.h"
#include "zo_kv.h"

#include <type_traits>

namespace {

constexpr int PG_W = 4;    // waves per workgroup
constexpr int PG_K = 32;   // keys per tile
constexpr float PG_LOW = -3.4028234663852886e38f;  // below every logit but -infinity

struct PagedArgs {
  KvArgs kv;
  const void* Q;
  void* O;
  long long ldq, ldo;
  int group, nsplit, tiles;           // heads per K/V head; splits; row tiles per (sequence, K/V head)
  int rt_rows, prows;                 // rows of a tile; those of them that partial results have room for
  int min_keys;                       // a split's keys at the least
  float scale_log2;                   // log2(e) / sqrt(dh)
  float* part;                        // nsplit > 1: O of a split, unnormalised, per row
  float2* stat;                       // its (maximum, sum)
};

// The splits that a range of `keys` keys is cut into, in whole tiles of `tile` keys.
__device__ __forceinline__ int splits_of(const PagedArgs& a, int keys) {
  return min(a.nsplit, max(1, (keys + a.min_keys - 1) / a.min_keys));
}

// What a row tile covers: rows [row0, row0 + nrows) of its (sequence, K/V head), keys [0, kend).
struct RowTile {
  KvSpan sp;
  int row0, nrows, kend;
};
__device__ __forceinline__ RowTile row_tile(const PagedArgs& a, int s, int rt) {
  RowTile t;
  t.sp = kv_span(a.kv, s);
  t.row0 = rt * a.rt_rows;
  const int all = min(t.sp.n, a.kv.max_q) * a.group;
  t.nrows = min(a.rt_rows, all - t.row0);
  t.kend = 0;
  if (t.nrows > 0) {
    const int last = t.sp.len - t.sp.n + (t.row0 + t.nrows - 1) / a.group;  // the last row's position
    if (a.kv.bad_flag && last >= kv_cap(a.kv)) *a.kv.bad_flag = 1;
    t.kend = max(0, min(last + 1, kv_cap(a.kv)));
  }
  return t;
}

// The pages of 64 runs of 16 keys, one per lane, from run r0 on; -1 for runs from `rend` on and for bad
// pages, which are not read: their keys and values (and scales) are 0.  `bad`: the first position of a
// bad page.
template <bool E8>
struct Pages {
  int page;
  float ks, vs;
  __device__ __forceinline__ void load(const PagedArgs& a, int s, int kvh, int r0, int rend, int lane, int& bad) {
    const int r = r0 + lane;
    page = -1;
    if (r < rend) {
      page = kv_page(a.kv, s, r >> (a.kv.log2ps - 4));
      if (page < 0) bad = min(bad, r * 16);
    }
    if constexpr (E8) {
      ks = page < 0 ? 0.f : a.kv.ks[(size_t)page * a.kv.kv_heads + kvh];
      vs = page < 0 ? 0.f : a.kv.vs[(size_t)page * a.kv.kv_heads + kvh];
    }
  }
};

__device__ __forceinline__ float lane_f(float v, int l) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l));
}

// Eight e4m3 codes as 16-bit values (exact).
template <bool F16>
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi) {
  if constexpr (F16)
    return (u32x4){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true))};
  else
    return (u32x4){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true))};
}

// Marks the top bit of every value (8-bit code, or 16-bit value) of a word that is an infinity or a NaN:
// one added to an exponent of all ones (a code of all ones) carries into the sign's place.
template <bool F16, bool E8>
__device__ __forceinline__ uint32_t odd_bits(u32x4 v) {
  constexpr uint32_t M = E8 ? 0x7f7f7f7fu : F16 ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t ONE = E8 ? 0x01010101u : F16 ? 0x04000400u : 0x00800080u;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (v[i] & M) + ONE;
  return any & (E8 ? 0x80808080u : 0x80008000u);
}

// A result o / l of a row at position p, from unnormalised sums: 0 where it has no keys, NaN where it
// attends to a position from `bad` on.
__device__ __forceinline__ float row_result(float o, float inv, int p, int bad) {
  return p < 0 ? 0.f : p >= bad ? __builtin_nanf("") : o * inv;
}

template <bool F16>
__device__ __forceinline__ void store4(uint16_t* dst, const float* y) {
  *(u32x2*)dst = F16 ? (u32x2){pack_f16x2(y[0], y[1]), pack_f16x2(y[2], y[3])}
                     : (u32x2){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

template <bool F16, bool E8, int DH, int NG>
__global__ __launch_bounds__(64 * PG_W, 2) void k_paged_rows(PagedArgs a) {
  constexpr int NT = PG_K / 16;            // 16-key tiles
  constexpr int KS = DH / 32;              // k steps of Q K^T
  constexpr int DT = DH / 16;              // 16-dim tiles of O
  constexpr int EB = E8 ? 1 : 2;           // bytes of a cached value
  constexpr int KV4 = 16 * DH * EB / 1024;  // 16-byte words per lane of 16 keys
  constexpr int VROW = DH + 16;            // LDS row of V (16-bit elements), padded for the transposed reads
  constexpr bool PF16 = F16 && !E8;        // type of the P V product
  constexpr float SHIFT = PF16 ? 12.f : 0.f;  // P = 2^(.. + SHIFT): keeps fp16 low parts normal
  constexpr int OROW = DH + 4;             // LDS row of the joined O (fp32)
  constexpr int VBYTES = PG_W * PG_K * VROW * 2, OBYTES = PG_W * 16 * NG * OROW * 4;
  __shared__ __attribute__((aligned(16))) char lds[VBYTES > OBYTES ? VBYTES : OBYTES];
  __shared__ float2 stats[PG_W][16 * NG];
  __shared__ int bads[PG_W];

  int w = blockIdx.x;
  const int split = w % a.nsplit;
  w /= a.nsplit;
  const int rt = w % a.tiles;
  w /= a.tiles;
  const int kvh = w % a.kv.kv_heads, s = w / a.kv.kv_heads;
  const RowTile rtile = row_tile(a, s, rt);
  if (rtile.nrows <= 0) return;
  const int nsp = splits_of(a, rtile.kend);
  if (split >= nsp) return;
  const int ntiles = (rtile.kend + PG_K - 1) / PG_K;
  const int t0 = (int)((long long)ntiles * split / nsp), t1 = (int)((long long)ntiles * (split + 1) / nsp);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int p0 = rtile.sp.len - rtile.sp.n;  // position of the sequence's row 0

  // This lane's queries (one per group) and their rows, in the order of K's fragments: lane group g's
  // step kk is dims 32 kk + 8 g; with 8-bit keys (16 per 16-byte word) 16 (g + 4 (kk / 2)) + 8 (kk % 2).
  int pos[NG];
  bf16x8 qf[NG][KS];
#pragma unroll
  for (int gq = 0; gq < NG; ++gq) {
    const int r = rtile.row0 + min(16 * gq + l16, rtile.nrows - 1);
    const int tok = r / a.group;
    pos[gq] = p0 + tok;
    const uint16_t* qp = (const uint16_t*)a.Q + (size_t)(rtile.sp.r0 + tok) * a.ldq + (size_t)(kvh * a.group + r % a.group) * DH;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
      qf[gq][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + (E8 ? 16 * (g + 4 * (kk >> 1)) + 8 * (kk & 1) : 32 * kk + 8 * g)));
  }
  const int pfirst = p0 + rtile.row0 / a.group;  // the tile's first position

  f32x4 o[NG][DT];
  float mrow[NG], lsum[NG];
#pragma unroll
  for (int gq = 0; gq < NG; ++gq) {
#pragma unroll
    for (int t = 0; t < DT; ++t) o[gq][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    mrow[gq] = PG_LOW;
    lsum[gq] = 0.f;
  }
  int bad = kv_cap(a.kv);
  uint16_t* const vs = (uint16_t*)lds + wave * PG_K * VROW;
  const int rend = (rtile.kend + 15) >> 4;
  const size_t head_bytes = (size_t)DH * EB << a.kv.log2ps;

  // The bytes of 16 keys (run r) of K or V.
  auto run_at = [&](const void* base, int page, int r) {
    return (const char*)base + ((size_t)page * a.kv.kv_heads + kvh) * head_bytes +
           (size_t)(r & ((1 << (a.kv.log2ps - 4)) - 1)) * (16 * DH * EB);
  };
  Pages<E8> pg;
  u32x4 kreg[NT][KV4], vreg[NT][KV4];
  auto load_k = [&](int tile, int lane0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int page = __builtin_amdgcn_readlane(pg.page, lane0 + t);
      const char* p = run_at(a.kv.K, page, NT * tile + t);
#pragma unroll
      for (int c = 0; c < KV4; ++c)
        kreg[t][c] = page < 0 ? (u32x4){0, 0, 0, 0} : *(const u32x4*)(p + l16 * DH * EB + 16 * g + 64 * c);
    }
  };
  auto load_v = [&](int tile, int lane0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int page = __builtin_amdgcn_readlane(pg.page, lane0 + t);
      const char* p = run_at(a.kv.V, page, NT * tile + t);
#pragma unroll
      for (int c = 0; c < KV4; ++c)
        vreg[t][c] = page < 0 ? (u32x4){0, 0, 0, 0} : *(const u32x4*)(p + 16 * lane + 1024 * c);
    }
  };

  int have = t0;  // pg holds the runs of tiles have .. have + 64 / NT - 1
  if (t0 + wave < t1) pg.load(a, s, kvh, NT * have, rend, lane, bad);
  for (int tile = t0 + wave; tile < t1; tile += PG_W) {
    if (tile >= have + 64 / NT) {
      have += 64 / NT;
      pg.load(a, s, kvh, NT * have, rend, lane, bad);
    }
    const int lane0 = NT * (tile - have);
    load_k(tile, lane0);
    load_v(tile, lane0);
    const int k0 = tile * PG_K;
    f32x4 st[NG][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int gq = 0; gq < NG; ++gq) st[gq][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        bf16x8 kf;
        if constexpr (E8) {
          const u32x4 x = kreg[t][kk >> 1];
          kf = __builtin_bit_cast(bf16x8, (kk & 1) ? widen8<F16>(x[2], x[3]) : widen8<F16>(x[0], x[1]));
        } else {
          kf = __builtin_bit_cast(bf16x8, kreg[t][kk]);
        }
#pragma unroll
        for (int gq = 0; gq < NG; ++gq) st[gq][t] = mfma16<F16>(kf, qf[gq][kk], st[gq][t]);
      }
      if constexpr (E8) {
        const float ks = lane_f(pg.ks, lane0 + t);
#pragma unroll
        for (int gq = 0; gq < NG; ++gq) st[gq][t] *= ks;
      }
    }
    // Keys that a row does not see; those behind the sequence are also cleared from V, where they may be
    // NaN.
    const bool mask = k0 + PG_K > pfirst + 1;
    uint32_t odd = 0;  // V of the tile is not finite
    if (mask) {
#pragma unroll
      for (int gq = 0; gq < NG; ++gq)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k0 + 16 * t + 4 * g + i > pos[gq]) st[gq][t][i] = -INFINITY;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < KV4; ++c) {
        constexpr int PER = 16 / EB, CPR = DH / PER;  // values of a word, words of a row
        const int x = lane + 64 * c, key = 16 * t + x / CPR, col = PER * (x % CPR);
        u32x4 v = vreg[t][c];
        if (k0 + key >= rtile.kend) v = (u32x4){0, 0, 0, 0};
        odd |= odd_bits<F16, E8>(v);
        uint16_t* dst = &vs[key * VROW + col];
        if constexpr (E8) {
          *(u32x4*)dst = widen8<false>(v[0], v[1]);
          *(u32x4*)(dst + 8) = widen8<false>(v[2], v[3]);
        } else {
          *(u32x4*)dst = v;
        }
      }
    // Online softmax: P = 2^((s - m) scale + SHIFT), the difference of the raw logits first, so that it
    // is exact near the maximum at any magnitude; m moves when a logit is more than 2^3 above it.
    bf16x8 bh[NT / 2][NG], bl[NT / 2][NG];
#pragma unroll
    for (int gq = 0; gq < NG; ++gq) {
      float tmax = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, st[gq][t][i]);
      tmax = max_groups(tmax);
      const float m = mrow[gq];
      if (__ballot((tmax - m) * a.scale_log2 > 3.f) != 0) {
        const float mnew = fmaxf(m, tmax);
        const float alpha = __builtin_amdgcn_exp2f((m - mnew) * a.scale_log2);
        mrow[gq] = mnew;
        lsum[gq] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[gq][t] *= alpha;
      }
#pragma unroll
      for (int c = 0; c < NT / 2; ++c) {
        u32x4 hp, lp;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int t = 2 * c + (x >> 1), i = 2 * (x & 1);
          float q0 = __builtin_amdgcn_exp2f(fmaf(st[gq][t][i] - mrow[gq], a.scale_log2, SHIFT));
          float q1 = __builtin_amdgcn_exp2f(fmaf(st[gq][t][i + 1] - mrow[gq], a.scale_log2, SHIFT));
          lsum[gq] += q0 + q1;
          if constexpr (E8) {
            const float vsc = lane_f(pg.vs, lane0 + t);
            q0 *= vsc;
            q1 *= vsc;
          }
          const uint32_t h = cvt_pk<PF16>(q0, q1);
          hp[x] = h;
          lp[x] = cvt_pk<PF16>(q0 - unpk<PF16>(h, 0), q1 - unpk<PF16>(h, 1));
        }
        bh[c][gq] = __builtin_bit_cast(bf16x8, hp);
        bl[c][gq] = __builtin_bit_cast(bf16x8, lp);
      }
    }
    if (__builtin_expect(__ballot(odd != 0) != 0, 0)) {
      // 0 times such a value is NaN, and hi and lo parts of P may have opposite signs: a row must not meet the
      // keys that it does not see, not even with P = 0, nor an infinity twice.  The tile's keys one by one,
      // in fp32.
#pragma unroll
      for (int gq = 0; gq < NG; ++gq)
#pragma unroll
        for (int x = 0; x < 4 * NT; ++x) {
          const int t = x >> 2, i = x & 3;
          const uint32_t hw = __builtin_bit_cast(u32x4, bh[t >> 1][gq])[2 * (t & 1) + (i >> 1)];
          const uint32_t lw = __builtin_bit_cast(u32x4, bl[t >> 1][gq])[2 * (t & 1) + (i >> 1)];
          const float pk = unpk<PF16>(hw, i & 1) + unpk<PF16>(lw, i & 1);
          for (int gg = 0; gg < 4; ++gg) {
            const float q = __shfl(pk, l16 + 16 * gg, 64);
            const int key = 16 * t + 4 * gg + i;
            if (k0 + key <= pos[gq]) {
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                const u32x2 v = *(const u32x2*)&vs[key * VROW + 16 * d + 4 * g];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[gq][d][e] = fmaf(q, unpk<PF16>(v[e >> 1], e & 1), o[gq][d][e]);
              }
            }
          }
        }
      continue;
    }
    // Lane group g's k slots are keys 32 c + 4 g + (0..3) and 32 c + 16 + 4 g + (0..3).
#pragma unroll
    for (int c = 0; c < NT / 2; ++c) {
      const uint16_t* vb = &vs[(32 * c + 4 * g + (l16 >> 2)) * VROW + 4 * (l16 & 3)];
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const u32x2 v0 = ds_read_tr(vb + 16 * t), v1 = ds_read_tr(vb + 16 * VROW + 16 * t);
        const bf16x8 af = __builtin_bit_cast(bf16x8, (u32x4){v0[0], v0[1], v1[0], v1[1]});
#pragma unroll
        for (int gq = 0; gq < NG; ++gq) {
          o[gq][t] = mfma16<PF16>(af, bh[c][gq], o[gq][t]);
          o[gq][t] = mfma16<PF16>(af, bl[c][gq], o[gq][t]);
        }
      }
    }
  }

  // The waves' results through LDS: O as rows of fp32, (maximum, sum) per row, the first bad position.
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) bad = min(bad, __shfl_xor(bad, off, 64));
  __syncthreads();  // the V tiles share the memory
  float* const os = (float*)lds;
#pragma unroll
  for (int gq = 0; gq < NG; ++gq) {
    float l = lsum[gq] + __shfl_xor(lsum[gq], 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) stats[wave][16 * gq + l16] = make_float2(mrow[gq], l);
#pragma unroll
    for (int t = 0; t < DT; ++t) *(f32x4*)&os[(size_t)(wave * 16 * NG + 16 * gq + l16) * OROW + 16 * t + 4 * g] = o[gq][t];
  }
  if (lane == 0) bads[wave] = bad;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PG_W; ++i) bad = min(bad, bads[i]);
  if (bad < kv_cap(a.kv) && threadIdx.x == 0 && a.kv.bad_flag) *a.kv.bad_flag = 1;
  constexpr int D4 = DH / 4;
  for (int x = threadIdx.x; x < rtile.nrows * D4; x += 64 * PG_W) {
    const int row = x / D4, d = 4 * (x % D4);
    float m = PG_LOW;
#pragma unroll
    for (int i = 0; i < PG_W; ++i) m = fmaxf(m, stats[i][row].x);
    float l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PG_W; ++i) {
      const float f = __builtin_amdgcn_exp2f((stats[i][row].x - m) * a.scale_log2);
      const f32x4 v = *(const f32x4*)&os[(size_t)(i * 16 * NG + row) * OROW + d];
      l += f * stats[i][row].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += f * v[e];
    }
    const int r = rtile.row0 + row, tok = r / a.group, p = p0 + tok;
    if (nsp == 1) {
      const float inv = 1.f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = row_result(y[e], inv, p, bad);
      store4<F16>((uint16_t*)a.O + (size_t)(rtile.sp.r0 + tok) * a.ldo + (size_t)(kvh * a.group + r % a.group) * DH + d, y);
    } else {
      // A split that met a bad page leaves NaN, which the join keeps.
      const size_t at = ((((size_t)s * a.kv.kv_heads + kvh) * a.tiles + rt) * a.nsplit + split) * a.prows + row;
      *(f32x4*)&a.part[at * DH + d] = (f32x4){y[0], y[1], y[2], y[3]};
      if (d == 0) a.stat[at] = make_float2(m, p >= bad ? __builtin_nanf("") : l);
    }
  }
}

// Joins the splits of a row: O = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i.  One workgroup per row; its
// 256 / (DH / 4) teams take the splits in turn.
template <bool F16, int DH>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  constexpr int D4 = DH / 4, TEAMS = 256 / D4;
  __shared__ f32x4 acc[TEAMS][D4];
  __shared__ float2 st[TEAMS];
  int w = blockIdx.x;
  const int row = w % a.prows;
  w /= a.prows;
  const int rt = w % a.tiles;
  w /= a.tiles;
  const int kvh = w % a.kv.kv_heads, s = w / a.kv.kv_heads;
  const RowTile rtile = row_tile(a, s, rt);
  if (row >= rtile.nrows) return;
  const int nsp = splits_of(a, rtile.kend);
  if (nsp == 1) return;  // written already
  const int team = threadIdx.x / D4, d = 4 * (threadIdx.x % D4);
  const size_t base = (((size_t)s * a.kv.kv_heads + kvh) * a.tiles + rt) * a.nsplit;
  float m = PG_LOW, l = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i = team; i < nsp; i += TEAMS) {
    const size_t at = (base + i) * a.prows + row;
    const float2 ml = a.stat[at];
    const f32x4 v = *(const f32x4*)&a.part[at * DH + d];
    const float mn = fmaxf(m, ml.x);
    const float f = __builtin_amdgcn_exp2f((m - mn) * a.scale_log2), h = __builtin_amdgcn_exp2f((ml.x - mn) * a.scale_log2);
    l = l * f + ml.y * h;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = y[e] * f + v[e] * h;
    m = mn;
  }
  acc[team][threadIdx.x % D4] = y;
  if (d == 0) st[team] = make_float2(m, l);
  __syncthreads();
  if (team) return;
  float mx = PG_LOW;
#pragma unroll
  for (int i = 0; i < TEAMS; ++i) mx = fmaxf(mx, st[i].x);
  float o[4] = {0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int i = 0; i < TEAMS; ++i) {
    const float f = __builtin_amdgcn_exp2f((st[i].x - mx) * a.scale_log2);
    l += f * st[i].y;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += f * acc[i][threadIdx.x][e];
  }
  const int r = rtile.row0 + row, tok = r / a.group, p = rtile.sp.len - rtile.sp.n + tok;
  const float inv = 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = row_result(o[e], inv, p, 0x7fffffff);
  store4<F16>((uint16_t*)a.O + (size_t)(rtile.sp.r0 + tok) * a.ldo + (size_t)(kvh * a.group + r % a.group) * DH + d, o);
}

}  // namespace

int zo_paged_attention_launch(const KvArgs& kv, const void* Q, long long ldq, void* O, long long ldo, void* ws,
                              hipStream_t stream, size_t* ws_needed) {
  PagedArgs a;
  a.kv = kv;
  a.Q = Q;
  a.O = O;
  a.ldq = ldq;
  a.ldo = ldo;
  a.group = kv.heads / kv.kv_heads;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)kv.dh);
  a.rt_rows = 16;
  const long long all_rows = (long long)kv.max_q * a.group;
  a.prows = (int)(all_rows < a.rt_rows ? all_rows : a.rt_rows);
  const long long tiles = (all_rows + a.rt_rows - 1) / a.rt_rows;
  const long long units = (long long)kv.nseq * kv.kv_heads * tiles;
  const long long keys = (long long)kv.max_pages << kv.log2ps;
  a.min_keys = 256;
  const long long most = (keys + a.min_keys - 1) / a.min_keys;
  long long split = 1024 / units;
  if (split < (keys + 2047) / 2048) split = (keys + 2047) / 2048;
  if (split > 64) split = 64;
  if (split > most) split = most;
  if (split < 1) split = 1;
  if (tiles > 0x7fffffffLL || units * split > 0x7fffffffLL || (split > 1 && units * a.prows > 0x7fffffffLL)) {
    zo_set_error("paged_attention: too many workgroups (%lld)", units * split);
    return ZO_ERR_UNSUPPORTED;
  }
  a.tiles = (int)tiles;
  a.nsplit = (int)split;
  WsCarver c(ws);
  const size_t prows = split > 1 ? (size_t)units * split * a.prows : 0;
  a.part = (float*)c.take(prows * kv.dh * 4);
  a.stat = (float2*)c.take(prows * 8);
  if (ws_needed) {
    *ws_needed = c.off;
    return ZO_OK;
  }
  const dim3 grid((unsigned)(units * split)), block(64 * PG_W);
  const bool f16 = kv.dtype == ZO_F16;
#define ZO_ROWS(F, E, D) hipLaunchKernelGGL((k_paged_rows<F, E, D, 1>), grid, block, 0, stream, a)
#define ZO_ROWS_D(F, E) \
  if (kv.dh == 64) ZO_ROWS(F, E, 64); \
  else ZO_ROWS(F, E, 128)
  if (kv.e8) {
    if (f16) { ZO_ROWS_D(true, true); } else { ZO_ROWS_D(false, true); }
  } else {
    if (f16) { ZO_ROWS_D(true, false); } else { ZO_ROWS_D(false, false); }
  }
#undef ZO_ROWS_D
#undef ZO_ROWS
  int st = zo_hip_status(hipGetLastError(), "k_paged_rows");
  if (st != ZO_OK || split == 1) return st;
  const dim3 jgrid((unsigned)(units * a.prows));
  if (f16) {
    if (kv.dh == 64) hipLaunchKernelGGL((k_paged_join<true, 64>), jgrid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_paged_join<true, 128>), jgrid, dim3(256), 0, stream, a);
  } else {
    if (kv.dh == 64) hipLaunchKernelGGL((k_paged_join<false, 64>), jgrid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_paged_join<false, 128>), jgrid, dim3(256), 0, stream, a);
  }
  return zo_hip_status(hipGetLastError(), "k_paged_join");
}
