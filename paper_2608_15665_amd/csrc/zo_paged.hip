// Causal attention over a paged key/value cache: few queries (a token, some drafted tokens, a piece
// of a prompt) against many keys.
//
// The queries of the heads that share a key/value head read the same keys, so a workgroup's rows are
// (token, head of the group) pairs of one key/value head: row t G + j is head j of the group at the
// sequence's new token t.  Softmax in one pass over the keys: a running maximum m, P = 2^((s - m) scale),
// a running sum of P and of P V, both scaled when m moves (by more than 2^3).
//
// k_paged_rows, for rows that read their keys and little else (up to 32): a workgroup of 4
// waves takes 16 NG rows and a range of the keys; its waves take the range's tiles (as many bytes each: 32 keys of 16
// bits, 64 of 8) in turn, each with a softmax of its own, and join their results in LDS at the end.  K goes from
// global memory straight into the fragments, a tile ahead.  Ranges of one sequence (nsplit > 1) are joined by
// k_paged_join.  Bound by HBM: 61 tokens with up to 8192 keys each, 40 query heads to 8, 198 us for 1.09 GB (5.5 TB/s,
// where a kernel that only reads reaches 6.0); one token, 131072 keys, 100 us for 0.54 GB with its join; 8-bit,
// 61 tokens, 112 us for 0.54 GB.
// k_paged_tile, for more rows: 4 waves of 32 rows share tiles of 64 keys in LDS.  Bound by the MFMAs and the
// exponentials between them: pieces of up to 1000 tokens of 4 sequences over up to 7000 keys, 330 us, 657 TFLOP/s of
// visible pairs (986 with the low parts), where a large matrix product reaches 1567; 8-bit pieces by the vector instructions that widen the codes.
//
// Products as in the causal attention of whole sequences:
//   S^T = K Q^T   (16 x 16 x 32 MFMA; A = K rows)
//   O^T += V^T P^T, V^T's fragments by transposed reads of a row-major V tile in LDS; P as a hi + lo
//   16-bit pair.
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
constexpr int PG_K8 = 64;  // and of 8-bit caches, as many bytes (61 sequences of up to 8192 keys: 121 -> 113 us)
constexpr float PG_LOW = -3.4028234663852886e38f;  // below every logit but -infinity

struct PagedArgs {
  KvArgs kv;
  const void* Q;
  void* O;
  long long ldq, ldo;
  int group, nsplit, tiles;           // heads per K/V head; splits; row tiles per (sequence, K/V head)
  int rt_rows, prows;                 // rows of a tile; those of them that partial results have room for
  int min_keys;                       // a split's keys at the least
  unsigned wgs;                       // workgroups of the launch
  uint32_t inv_group;                 // 2^32 / group, rounded up past a whole one; 0: group is 1
  float scale_log2;                   // log2(e) / sqrt(dh)
  float* part;                        // nsplit > 1: O of a split, unnormalised, per row
  float2* stat;                       // its (maximum, sum)
};

// The splits that a range of `keys` keys is cut into.
__device__ __forceinline__ int splits_of(const PagedArgs& a, int keys) {
  return keys <= 512 ? 1 : min(a.nsplit, max(1, (keys + a.min_keys - 1) / a.min_keys));
}

// The sequence that is i-th when every 64 consecutive ones are ordered by their lengths, the longest first
// (workgroups start in that order, so that the long ones are not the last to end), and its rows and length: the
// loads of all lanes' sequences go out together, and the one that it is comes from its lane.
__device__ __forceinline__ int by_length(const KvArgs& a, int i, int lane, KvSpan& sp) {
  const int s0 = i & ~63, n = min(64, a.nseq - s0);
  const int mine = s0 + min(lane, n - 1);
  const KvSpan own = kv_span(a, mine);
  int rank = 0;
  for (int j = 0; j < n; ++j) {
    const int other = __builtin_amdgcn_readlane(own.len, j);
    rank += other > own.len || (other == own.len && j < lane);
  }
  const int l = __builtin_ctzll(__ballot(lane < n && rank == (i & 63)));
  sp.r0 = __builtin_amdgcn_readlane(own.r0, l);
  sp.n = __builtin_amdgcn_readlane(own.n, l);
  sp.len = __builtin_amdgcn_readlane(own.len, l);
  return s0 + l;
}

// What a row tile covers: rows [row0, row0 + nrows) of its (sequence, K/V head), keys [0, kend).  Row i of the tile
// is token tok(i) of the sequence's new ones and head i + rem - group (tok(i) - tok0) of the group.
struct RowTile {
  KvSpan sp;
  int row0, nrows, kend;
  int tok0, rem, group;
  uint32_t inv;
  // (row0 + i) / group by a product: i + rem < 2^32 / group, where the rounded inverse is exact.
  __device__ __forceinline__ int tok(int i) const { return tok0 + (inv ? (int)__umulhi((uint32_t)(i + rem), inv) : i); }
  __device__ __forceinline__ int head(int i) const { return i + rem - group * (tok(i) - tok0); }
  __device__ __forceinline__ int pos(int i) const { return sp.len - sp.n + tok(i); }
};
__device__ __forceinline__ RowTile row_tile(const PagedArgs& a, const KvSpan& sp, int rt) {
  RowTile t;
  t.sp = sp;
  t.row0 = rt * a.rt_rows;
  t.group = a.group;
  t.inv = a.inv_group;
  t.tok0 = t.row0 / a.group;
  t.rem = t.row0 - t.tok0 * a.group;
  const int all = min(sp.n, a.kv.max_q) * a.group;
  t.nrows = min(a.rt_rows, all - t.row0);
  t.kend = 0;
  if (t.nrows > 0) {
    const int last = t.pos(t.nrows - 1);  // the last row's position
    if (a.kv.bad_flag && last >= kv_cap(a.kv)) *a.kv.bad_flag = 1;
    t.kend = max(0, min(last + 1, kv_cap(a.kv)));
  }
  return t;
}

// Where 64 runs of 16 keys lie in K (and, in the same place, in V), one per lane, from run r0 on: as a number of
// runs from the cache's start.  Runs from `rend` on, and those of bad pages, lie in page 0, which exists: their keys are
// masked (or their rows NaN) and their values cleared or, in a tile that is masked anyway, harmless; their
// scales are 0.  Without a branch at the load, the loads of a tile stay in flight together.
// `bad`: the first position of a bad page.
template <bool E8>
struct Runs {
  uint32_t run;
  float ks, vs;
  // Two steps, so that loads of several windows go out together: the table's entry, then the rest.
  __device__ __forceinline__ void fetch(const PagedArgs& a, int s, int r0, int lane) {
    const int j = min((r0 + lane) >> (a.kv.log2ps - 4), a.kv.max_pages - 1);
    run = a.kv.table[(size_t)s * a.kv.max_pages + j];
  }
  __device__ __forceinline__ void place(const PagedArgs& a, int kvh, int r0, int rend, int lane, int& bad) {
    const int r = r0 + lane, lr = a.kv.log2ps - 4;
    const bool used = r < rend && run < (uint32_t)a.kv.num_pages;
    if (r < rend && !used) bad = min(bad, r * 16);
    const uint32_t head = (used ? run : 0) * a.kv.kv_heads + kvh;
    run = (head << lr) + (r & ((1 << lr) - 1));
    if constexpr (E8) {
      ks = used ? a.kv.ks[head] : 0.f;
      vs = used ? a.kv.vs[head] : 0.f;
    }
  }
  template <int RUN>  // bytes of a run
  __device__ __forceinline__ size_t at(int l) const {
    return (size_t)(uint32_t)__builtin_amdgcn_readlane(run, l) * RUN;
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

// A pair of 16-bit values with infinities and NaN as 0.
template <bool F16>
__device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
  const uint32_t t = ((x & (F16 ? 0x7c007c00u : 0x7f807f80u)) + (F16 ? 0x04000400u : 0x00800080u)) & 0x80008000u;
  return x & ~((t - (t >> 15)) | t);
}

// V of a staged tile of `keys` keys is not finite somewhere.  0 times such a value is NaN, so a product with
// P = 0 would take it to rows that do not see the key (and a hi + lo pair may meet an infinity with opposite
// signs).  P V then runs on V without such values, and here they are added to the rows that do see them.
// at(key, d): where values d .. d + 3 of a key lie.  Of the keys the first is looked at in any case (a loop that may
// have no turn costs the caller registers).
template <bool F16, bool E8, int DT, int NG, class At>
__device__ __forceinline__ void add_odd_values(At at, int k0, int keys, int g, const int* pos, f32x4 (*o)[DT]) {
  int key = 0;
#pragma unroll 1
  do {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      u32x2 v;
      if constexpr (E8) {
        const u32x4 x = widen8<F16>(*(const uint32_t*)at(key, 16 * d + 4 * g), 0);
        v = (u32x2){x[0], x[1]};
      } else {
        v = *(const u32x2*)at(key, 16 * d + 4 * g);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = unpk<F16>(v[e >> 1], e & 1);
#pragma unroll
        for (int gq = 0; gq < NG; ++gq)
          if (k0 + key <= pos[gq] && !(fabsf(x) < INFINITY)) o[gq][d][e] += x;
      }
    }
  } while (++key < keys);
}

typedef int i32x2_t __attribute__((ext_vector_type(2)));
// ds_read_b64_tr_b8: within each 16-lane group, lane i reads 8 bytes D[i][0..7] at its own address, and lane j
// receives D[2 e + j / 8][j % 8] for e = 0..7.  With lanes 2 e and 2 e + 1 addressing the two halves of 16 columns
// of row r_e, lane j thus receives column j of rows r_0 .. r_7.
__device__ __forceinline__ u32x2 ds_read_tr8(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2_t*)p));
}

// Two fp32 values (0 or more) rounded down into a packed pair of 16-bit values.
template <bool F16>
__device__ __forceinline__ uint32_t cvt_down(float x, float y) {
  if constexpr (F16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));
  else
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
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
  constexpr int KT = E8 && NG == 1 ? PG_K8 : PG_K;  // keys per tile
  constexpr int NT = KT / 16;              // 16-key tiles
  constexpr int KS = DH / 32;              // k steps of Q K^T
  constexpr int DT = DH / 16;              // 16-dim tiles of O
  constexpr int EB = E8 ? 1 : 2;           // bytes of a cached value
  constexpr int KV4 = 16 * DH * EB / 1024;  // 16-byte words per lane of 16 keys
  constexpr int VROW = DH + 16;            // LDS row of V (16-bit elements), padded for the transposed reads
  constexpr bool PF16 = F16 && !E8;        // type of the P V product
  constexpr float SHIFT = PF16 ? 12.f : 0.f;  // P = 2^(.. + SHIFT): keeps fp16 low parts normal
  constexpr int OROW = DH + 4;             // LDS row of the joined O (fp32)
  constexpr int VBYTES = PG_W * KT * VROW * 2, OBYTES = PG_W * 16 * NG * OROW * 4;
  __shared__ __attribute__((aligned(16))) char lds[VBYTES > OBYTES ? VBYTES : OBYTES];
  __shared__ float2 stats[PG_W][16 * NG];
  __shared__ int bads[PG_W];

  if (kv_block() >= a.wgs) return;
  int w = kv_block();
  const int split = w % a.nsplit;
  w /= a.nsplit;
  const int rt = w % a.tiles;
  w /= a.tiles;
  const int kvh = w % a.kv.kv_heads;
  KvSpan sp;
  const int s = by_length(a.kv, w / a.kv.kv_heads, threadIdx.x & 63, sp);
  const RowTile rtile = row_tile(a, sp, rt);
  if (rtile.nrows <= 0) return;
  const int nsp = splits_of(a, rtile.kend);
  if (split >= nsp) return;
  const int ntiles = (rtile.kend + KT - 1) / KT;
  const int t0 = (int)((long long)ntiles * split / nsp), t1 = (int)((long long)ntiles * (split + 1) / nsp);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;

  // This lane's queries (one per group) and their rows, in the order of K's fragments: lane group g's
  // step kk is dims 32 kk + 8 g; with 8-bit keys (16 per 16-byte word) 16 (g + 4 (kk / 2)) + 8 (kk % 2).
  int pos[NG];
  bf16x8 qf[NG][KS];
#pragma unroll
  for (int gq = 0; gq < NG; ++gq) {
    const int i = min(16 * gq + l16, rtile.nrows - 1);
    pos[gq] = rtile.pos(i);
    const uint16_t* qp = (const uint16_t*)a.Q + (size_t)(rtile.sp.r0 + rtile.tok(i)) * a.ldq + (size_t)(kvh * a.group + rtile.head(i)) * DH;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
      qf[gq][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + (E8 ? 16 * (g + 4 * (kk >> 1)) + 8 * (kk & 1) : 32 * kk + 8 * g)));
  }
  const int pfirst = rtile.pos(0);  // the tile's first position

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
  uint16_t* const vs = (uint16_t*)lds + wave * KT * VROW;
  const int rend = (rtile.kend + 15) >> 4;

  // The run window at hand (64 runs, the tiles from `have` on) and the one after it, on its way.
  constexpr int WT = 64 / NT, RUN = 16 * DH * EB;
  Runs<E8> pg, pgn;
  u32x4 kreg[NT][KV4], vreg[NT][KV4];
  auto load_k = [&](int lane0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const char* p = (const char*)a.kv.K + pg.template at<RUN>(lane0 + t);
#pragma unroll
      for (int c = 0; c < KV4; ++c) kreg[t][c] = *(const u32x4*)(p + l16 * DH * EB + 16 * g + 64 * c);
    }
  };
  auto load_v = [&](int lane0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const char* p = (const char*)a.kv.V + pg.template at<RUN>(lane0 + t);
#pragma unroll
      for (int c = 0; c < KV4; ++c) vreg[t][c] = *(const u32x4*)(p + 16 * lane + 1024 * c);
    }
  };

  int have = t0;
  float ksc[NT], vsc[NT];  // 8-bit: the scales of the tile at hand
  auto scales = [&](int lane0) {
    if constexpr (E8) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        ksc[t] = lane_f(pg.ks, lane0 + t);
        vsc[t] = lane_f(pg.vs, lane0 + t);
      }
    }
  };
  if (t0 + wave < t1) {
    pg.fetch(a, s, NT * have, lane);
    pgn.fetch(a, s, NT * (have + WT), lane);
    pg.place(a, kvh, NT * have, rend, lane, bad);
    pgn.place(a, kvh, NT * (have + WT), rend, lane, bad);
    load_k(NT * wave);
    load_v(NT * wave);
  }
  for (int tile = t0 + wave; tile < t1; tile += PG_W) {
    scales(NT * (tile - have));
    // The wave's next tile: its K is on its way from the end of this one's S on, its V from the store of this
    // one's.
    const int next = tile + PG_W;
    const bool more = next < t1;
    if (more && next >= have + WT) {
      have += WT;
      pg = pgn;
      pgn.fetch(a, s, NT * (have + WT), lane);
      pgn.place(a, kvh, NT * (have + WT), rend, lane, bad);
    }
    const int lane0 = NT * (next - have);
    const int k0 = tile * KT;
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
#pragma unroll
        for (int gq = 0; gq < NG; ++gq) st[gq][t] *= ksc[t];
      }
    }
    if (more) load_k(lane0);
    // Keys that a row does not see; those behind the sequence are also cleared from V, where they may be
    // NaN.
    const bool mask = k0 + KT > pfirst + 1;
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
    if (more) load_v(lane0);
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
            q0 *= vsc[t];
            q1 *= vsc[t];
          }
          const uint32_t h = cvt_pk<PF16>(q0, q1);
          hp[x] = h;
          lp[x] = cvt_pk<PF16>(q0 - unpk<PF16>(h, 0), q1 - unpk<PF16>(h, 1));
        }
        bh[c][gq] = __builtin_bit_cast(bf16x8, hp);
        bl[c][gq] = __builtin_bit_cast(bf16x8, lp);
      }
    }
    // Lane group g's k slots are keys 32 c + 4 g + (0..3) and 32 c + 16 + 4 g + (0..3).
    auto pv = [&](bool clean) {
#pragma unroll
      for (int c = 0; c < NT / 2; ++c) {
        const uint16_t* vb = &vs[(32 * c + 4 * g + (l16 >> 2)) * VROW + 4 * (l16 & 3)];
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const u32x2 v0 = ds_read_tr(vb + 16 * t), v1 = ds_read_tr(vb + 16 * VROW + 16 * t);
          u32x4 av = {v0[0], v0[1], v1[0], v1[1]};
          if (clean)
            av = (u32x4){finite_pair<PF16>(av[0]), finite_pair<PF16>(av[1]), finite_pair<PF16>(av[2]), finite_pair<PF16>(av[3])};
          const bf16x8 af = __builtin_bit_cast(bf16x8, av);
#pragma unroll
          for (int gq = 0; gq < NG; ++gq) {
            o[gq][t] = mfma16<PF16>(af, bh[c][gq], o[gq][t]);
            o[gq][t] = mfma16<PF16>(af, bl[c][gq], o[gq][t]);
          }
        }
      }
    };
    const bool clean = __builtin_expect(__ballot(odd != 0) != 0, 0);
    if (clean) add_odd_values<PF16, false, DT, NG>([&](int key, int d) { return &vs[key * VROW + d]; }, k0, KT, g, pos, o);
    // Two copies of P V, without a branch at each fragment, where the registers allow it.
    if constexpr (NG == 1) {
      if (clean) pv(true);
      else pv(false);
    } else {
      pv(clean);
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
    const int p = rtile.pos(row);
    if (nsp == 1) {
      const float inv = 1.f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = row_result(y[e], inv, p, bad);
      store4<F16>((uint16_t*)a.O + (size_t)(rtile.sp.r0 + rtile.tok(row)) * a.ldo + (size_t)(kvh * a.group + rtile.head(row)) * DH + d, y);
    } else {
      // A split that met a bad page leaves NaN, which the join keeps.
      const size_t at = ((((size_t)s * a.kv.kv_heads + kvh) * a.tiles + rt) * a.nsplit + split) * a.prows + row;
      *(f32x4*)&a.part[at * DH + d] = (f32x4){y[0], y[1], y[2], y[3]};
      if (d == 0) a.stat[at] = make_float2(m, p >= bad ? __builtin_nanf("") : l);
    }
  }
}

// ---------------------------------------------------------------- many rows
constexpr int PT_NG = 2;                  // 16-row groups per wave
constexpr int PT_Q = 16 * PT_NG * PG_W;   // rows per workgroup
constexpr int PT_K = 64;                  // keys per tile
constexpr float PT_RAW = 1048576.f;       // maxima from here on (in log2 units) are subtracted from the logits
constexpr int PT_AHEAD = 2;               // LDS reads of a phase that go out before its first MFMA

// A workgroup of 4 waves takes PT_Q rows and a range of the keys.  Tiles of K and V come as stored (8-bit
// codes too) by direct global -> LDS loads, two of each: while tile n is worked on, V of tile n + 1 and K of
// tile n + 2 land, K of n + 1 has landed, and one barrier a tile is enough.  Tile n + 1's S runs under tile
// n's exponentials.  A load fills 1024 bytes of LDS, some rows of RB bytes; each such block is followed by a pad,
// and within a row the 16-byte chunks are permuted by an XOR with swz(row) in two bits, so that the 16 rows of a K
// fragment, and the 8 (8-bit: 16) rows of a transposed read of V, lie on different banks.  A read's address is then
// one of one (K) or four (V) per lane, the rest is an immediate offset.
// 8-bit tiles take 600 vector instructions of a wave beside its 96 MFMAs where 16-bit ones take 370 (128 widen the
// codes, which every wave does for itself, 64 apply the scales): 8 pieces of up to 256 tokens over up to 4096 keys,
// 32 heads, 142 us (16 bits: 120).  Four buffers of each instead of two, with the loads three tiles ahead, gained
// nothing (2 % slower), so it is not their latency.
// P enters its product as a hi + lo pair, as in k_paged_rows, so a row is as exact here as it is alone.  That is half as
// many MFMAs again: the pieces above took 114 us (8 bits) and 100 (16 bits) with P rounded once, which put an
// output off by up to 2^-8 (bf16) or 2^-11 (fp16) of the values it averages.
template <int RB>
__device__ __forceinline__ int swz(int r) {
  return RB == 256 ? r & 3 : RB == 128 ? (r >> 1) & 3 : (r >> 2) & 3;
}

template <bool F16, bool E8, int DH>
__global__ __launch_bounds__(64 * PG_W, 2) void k_paged_tile(PagedArgs a) {
  constexpr int NTH = 64 * PG_W;
  constexpr int KS = DH / 32, DT = DH / 16;
  constexpr int EB = E8 ? 1 : 2, RB = DH * EB;  // bytes of a cached value, of a row
  constexpr int CPR = RB / 16;                  // chunks of a row
  constexpr int KCH = PT_K * CPR / NTH;         // loads per thread and tile
  constexpr int RUN = 16 * RB, RPB = 1024 / RB;  // bytes of 16 keys, rows of a block of LDS
  constexpr int KBLK = 1024 + (RB == 64 ? 0 : 64), VBLK = 1024 + (E8 ? 32 : RB == 256 ? 128 : 0);
  constexpr int NBLK = PT_K / RPB;               // blocks of a tile
  constexpr int VX = E8 ? 1 : 2;                 // V's chunks are permuted one by one or in pairs
  constexpr bool PF16 = F16 && !E8;
  constexpr float PULL = F16 || E8 ? 1.f : 1.f + 0x1p-18f;  // P's factor (see probs)
  constexpr float SHIFT = PF16 ? 12.f : 0.f;
  constexpr int OROW = DH + 8;  // LDS row of the finished rows (16-bit elements)
  static_assert(16 * OROW * 2 <= NBLK * 1024, "16 finished rows of a wave fit a buffer");
  // Four arrays, and steps that know at compile time which they use: the compiler then sees that a tile's reads
  // do not meet the loads under way, and does not wait for those.
  __shared__ __attribute__((aligned(1024))) char Kb0[NBLK * KBLK], Kb1[NBLK * KBLK], Vb0[NBLK * VBLK],
      Vb1[NBLK * VBLK];
  __shared__ int bads[PG_W];

  // Workgroups are dealt to the 8 XCDs in turn.  Where the key heads are a multiple of 8, each XCD takes as many of
  // them, the longest sequence of all its heads first (8 sequences in pieces of up to 256 over up to 4096 keys, 32
  // heads: 120 us, head after head 152; 8-bit 142 and 192); else a contiguous range of (head, sequence) pairs.  The
  // row tiles that read one sequence's keys share its L2, and sequences of different lengths load the XCDs alike.
  const unsigned block = kv_block();
  if (block >= a.wgs) return;
  const int xcd = (int)(block & 7), hx = a.kv.kv_heads & 7 ? 0 : a.kv.kv_heads >> 3;
  int w = (int)(block >> 3);
  if (!hx) w += xcd * (int)(a.wgs >> 3) + min(xcd, (int)(a.wgs & 7));
  const int rt = a.tiles - 1 - w % a.tiles;  // the last rows see the most keys: they begin first
  w /= a.tiles;
  const int split = w % a.nsplit;
  w /= a.nsplit;
  const int kvh = hx ? xcd * hx + w % hx : w / a.kv.nseq;
  KvSpan sp;
  const int s = by_length(a.kv, hx ? w / hx : w % a.kv.nseq, threadIdx.x & 63, sp);
  const RowTile rtile = row_tile(a, sp, rt);
  if (rtile.nrows <= 0) return;
  const int nsp = splits_of(a, rtile.kend);
  if (split >= nsp) return;
  const int ntiles = (rtile.kend + PT_K - 1) / PT_K;
  const int t0 = (int)((long long)ntiles * split / nsp), t1 = (int)((long long)ntiles * (split + 1) / nsp);
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr0 = 16 * PT_NG * wave;  // the wave's first row in the tile

  Runs<E8> pg, pgn;
  int win = t0 >> 4;
  pg.fetch(a, s, 64 * win, lane);
  pgn.fetch(a, s, 64 * (win + 1), lane);
  // Rows as B operands of S^T, in the order of K's fragments (see k_paged_rows).
  int pos[PT_NG];
  bf16x8 qf[PT_NG][KS];
#pragma unroll
  for (int gq = 0; gq < PT_NG; ++gq) {
    const int i = min(wr0 + 16 * gq + l16, rtile.nrows - 1);
    pos[gq] = rtile.pos(i);
    const uint16_t* qp = (const uint16_t*)a.Q + (size_t)(rtile.sp.r0 + rtile.tok(i)) * a.ldq + (size_t)(kvh * a.group + rtile.head(i)) * DH;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
      qf[gq][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + (E8 ? 16 * (g + 4 * (kk >> 1)) + 8 * (kk & 1) : 32 * kk + 8 * g)));
  }
  // Positions of the wave's first and last row.
  const int wfirst = rtile.pos(min(wr0, rtile.nrows - 1));
  const int wlast = wr0 < rtile.nrows ? rtile.pos(min(wr0 + 16 * PT_NG, rtile.nrows) - 1) : -1;

  // P = 2^(s scale + b), b = SHIFT - m scale rounded: its rounding is the same factor for all of a row's P, and
  // from one maximum m to the next the exact b are subtracted.  Where m scale is so large that the rounding
  // could be whole powers of two (`raw`, of the wave, from then on), m is subtracted from the logits first and b
  // is SHIFT.
  f32x4 o[PT_NG][DT];
  float mrow[PT_NG], brow[PT_NG], lsum[PT_NG];  // lsum: of this lane's keys
  int raw = 0;
#pragma unroll
  for (int gq = 0; gq < PT_NG; ++gq) {
#pragma unroll
    for (int t = 0; t < DT; ++t) o[gq][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    lsum[gq] = 0.f;
    mrow[gq] = PG_LOW;
    brow[gq] = 0.f;
  }
  int bad = kv_cap(a.kv);
  const int rend = (rtile.kend + 15) >> 4;

  // Load c of this wave fills block 4 c + wave: rows RPB (4 c + wave) + lane / CPR, which lie in one run of 16 keys.
  // pg: the runs of tiles 16 win .. 16 win + 15, pgn those of the next 16.  K of a tile is loaded one tile before
  // V, which lies in the same place of its tensor.
  const int drow = (RPB * wave + lane / CPR) & 15;  // of every c
  const unsigned offk = (unsigned)(drow * RB + 16 * ((lane % CPR) ^ swz<RB>(drow)));
  const unsigned offv = (unsigned)(drow * RB + 16 * ((lane % CPR) ^ (VX * swz<RB>(drow))));
  float ksp = 0.f, vsp = 0.f;  // 8-bit: the scales of the window before pg's
  auto dma = [&](const void* base, int tile, unsigned off, char* dst, int blk) {
#pragma unroll
    for (int c = 0; c < KCH; ++c) {
      const char* at = (const char*)base + pg.template at<RUN>(4 * (tile & 15) + RPB * (PG_W * c + wave) / 16);
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)at, (short)0, RUN, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)(dst + (PG_W * c + wave) * blk), 16, off, 0, 0, 0);
    }
  };
  auto load_k = [&](int tile, char* dst) {
    if ((tile >> 4) != win) {
      win = tile >> 4;
      if constexpr (E8) {
        ksp = pg.ks;
        vsp = pg.vs;
      }
      pg = pgn;
      pgn.fetch(a, s, 64 * (win + 1), lane);
      pgn.place(a, kvh, 64 * (win + 1), rend, lane, bad);
    }
    dma(a.kv.K, tile, offk, dst, KBLK);
  };
  // V of the tile whose K was loaded last.
  auto load_v = [&](int tile, char* dst) { dma(a.kv.V, tile, offv, dst, VBLK); };
  // Everything that this wave loads has landed; with the barrier, that of all waves.
  auto landed = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
  };

  // Where this lane reads: fragment kk (8 bits: pair of fragments) of K's row 16 t + l16 at kat + 64 kk, row
  // blocks ahead; V's column 16 t of key 32 c + .. at vat[t % 4] and whole 4 t ahead.
  const int kat = l16 / RPB * KBLK + l16 % RPB * RB + 16 * (g ^ swz<RB>(l16));
  const int vrow = 4 * g + (E8 ? ((l16 >> 1) & 3) + 16 * (l16 >> 3) : l16 >> 2);
  int vat[4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
    vat[t] = vrow / RPB * VBLK + vrow % RPB * RB + 16 * VX * (t ^ swz<RB>(vrow)) + (E8 ? 0 : 16 * ((l16 >> 1) & 1)) + 8 * (l16 & 1);
  // S^T of the four runs of 16 keys of a staged K tile.
  auto qk = [&](const char* kb, f32x4 (*st)[4]) {
#pragma unroll
    for (int kk = 0; kk < KS; kk += E8 ? 2 : 1)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const char* p = kb + kat + 16 / RPB * KBLK * t + (E8 ? 32 * kk : 64 * kk);
        if (kk == 0) {
#pragma unroll
          for (int gq = 0; gq < PT_NG; ++gq) st[gq][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (E8) {
          const u32x4 x = *(const u32x4*)p;
          const bf16x8 k0 = __builtin_bit_cast(bf16x8, widen8<F16>(x[0], x[1])), k1 = __builtin_bit_cast(bf16x8, widen8<F16>(x[2], x[3]));
#pragma unroll
          for (int gq = 0; gq < PT_NG; ++gq) {
            st[gq][t] = mfma16<F16>(k0, qf[gq][kk], st[gq][t]);
            st[gq][t] = mfma16<F16>(k1, qf[gq][kk + 1], st[gq][t]);
          }
        } else {
          const bf16x8 kf = *(const bf16x8*)p;
#pragma unroll
          for (int gq = 0; gq < PT_NG; ++gq) st[gq][t] = mfma16<F16>(kf, qf[gq][kk], st[gq][t]);
        }
      }
  };
  // 8-bit: the scales of tile n's four runs, of keys or values.
  auto scales = [&](int n, float now, float before, float* out) {
#pragma unroll
    for (int t = 0; t < 4; ++t) out[t] = lane_f((n >> 4) == win ? now : before, 4 * (n & 15) + t);
  };
  auto scale_s = [&](int n, f32x4 (*st)[4]) {
    if constexpr (E8) {
      float ks[4];
      scales(n, pg.ks, ksp, ks);
#pragma unroll
      for (int gq = 0; gq < PT_NG; ++gq)
#pragma unroll
        for (int t = 0; t < 4; ++t) st[gq][t] *= ks[t];
    }
  };
  auto top_of = [&](f32x4 (*st)[4], float* tmax) {
#pragma unroll
    for (int gq = 0; gq < PT_NG; ++gq) {
      tmax[gq] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) tmax[gq] = fmaxf(tmax[gq], st[gq][t][i]);
      tmax[gq] = max_groups(tmax[gq]);
    }
  };
  // One tile: its softmax and P V from V's buffer vt, st being its S and tmax S's largest entries (of whole tiles).
  // NEXT: also the next tile's S (into sn, from K's buffer kb) and its tmax; such a tile lies wholly before the
  // workgroup's rows.
  auto tile = [&](auto NEXT, int n, const char* vt, const char* kb, f32x4 (*st)[4], f32x4 (*sn)[4], float* tmax) {
    constexpr bool next = decltype(NEXT)::value;
    const int k0 = PT_K * n;
    float vsc[4];
    if constexpr (E8) scales(n, pg.vs, vsp, vsc);
    if constexpr (!next) scale_s(n, st);
    bool clean = false;  // V of the tile is not finite
    int odds = 1;  // keys to look for such values in
    if (!next) {
      if (k0 + PT_K > wfirst + 1) {
#pragma unroll
        for (int gq = 0; gq < PT_NG; ++gq)
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (k0 + 16 * t + 4 * g + i > pos[gq]) st[gq][t][i] = -INFINITY;
      }
      // What is behind the wave's last row (slots behind the sequence among it, which may hold anything) only has to
      // be kept out of the product.
      const int keys = min(PT_K, wlast + 1 - k0);
      uint32_t odd = 0, seen = 0;
#pragma unroll 4
      for (int x = 0; x < NBLK; ++x) {
        const uint32_t b = odd_bits<PF16, E8>(*(const u32x4*)(vt + VBLK * x + 16 * lane));
        odd |= b;
        seen |= RPB * x + lane / CPR < keys ? b : 0;
      }
      if (__ballot(seen != 0) != 0) odds = keys;
      clean = __ballot(odd != 0) != 0;
    }
    if constexpr (!next) top_of(st, tmax);
#pragma unroll
    for (int gq = 0; gq < PT_NG; ++gq) {
      const float m = mrow[gq];
      if (__builtin_expect(__ballot((tmax[gq] - m) * a.scale_log2 > 3.f) != 0, 0)) {
        const float mnew = fmaxf(m, tmax[gq]), b = brow[gq];
        const bool was = raw != 0;
        raw |= __ballot(mnew > PG_LOW && !(fabsf(mnew * a.scale_log2) < PT_RAW)) != 0;
        const float bnew = raw ? SHIFT : fmaf(-mnew, a.scale_log2, SHIFT);
        // 2^(what P = 1 now stands for, relative to before)
        float d = was ? (m - mnew) * a.scale_log2 : raw ? SHIFT - fmaf(mnew, a.scale_log2, b) : bnew - b;
        if (m == PG_LOW) d = mnew == PG_LOW ? 0.f : -INFINITY;
        const float alpha = __builtin_amdgcn_exp2f(d);
        mrow[gq] = mnew;
        brow[gq] = bnew;
        lsum[gq] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[gq][t] *= alpha;
        if (raw && !was) {
          // the other rows of the wave, from their b to their maximum
#pragma unroll
          for (int x = 0; x < PT_NG; ++x)
            if (x != gq) {
              const float f = mrow[x] == PG_LOW ? 1.f : __builtin_amdgcn_exp2f(SHIFT - fmaf(mrow[x], a.scale_log2, brow[x]));
              brow[x] = SHIFT;
              lsum[x] *= f;
#pragma unroll
              for (int t = 0; t < DT; ++t) o[x][t] *= f;
            }
        }
      }
    }
    if (__builtin_expect(raw, 0)) {
#pragma unroll
      for (int gq = 0; gq < PT_NG; ++gq)
#pragma unroll
        for (int t = 0; t < 4; ++t) st[gq][t] -= mrow[gq];
    }
    // P as a hi + lo pair.  An infinity of V (8-bit codes have none) times such a pair is NaN unless lo is positive
    // as well.  Where rows see all of a tile, which is not searched for infinities, it is: hi is rounded down, and
    // lo then holds PULL times P less hi (bf16; the sum of P gets the same factor), or its last bit is set (fp16,
    // at most 2^-20 of P or 2^-24).
    bf16x8 bh[2][PT_NG], bl[2][PT_NG];
    auto probs = [&](int c) {
#pragma unroll
      for (int gq = 0; gq < PT_NG; ++gq) {
        u32x4 hp, lp;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int t = 2 * c + (x >> 1), i = 2 * (x & 1);
          float q0 = __builtin_amdgcn_exp2f(fmaf(st[gq][t][i], a.scale_log2, brow[gq]));
          float q1 = __builtin_amdgcn_exp2f(fmaf(st[gq][t][i + 1], a.scale_log2, brow[gq]));
          lsum[gq] += q0 + q1;
          if constexpr (E8) {
            q0 *= vsc[t];
            q1 *= vsc[t];
          }
          hp[x] = E8 ? cvt_pk<PF16>(q0, q1) : cvt_down<PF16>(q0, q1);
          lp[x] = cvt_pk<PF16>(fmaf(q0, PULL, -unpk<PF16>(hp[x], 0)), fmaf(q1, PULL, -unpk<PF16>(hp[x], 1)));
          if constexpr (PF16 && next) lp[x] |= 0x00010001u;
        }
        bh[c][gq] = __builtin_bit_cast(bf16x8, hp);
        bl[c][gq] = __builtin_bit_cast(bf16x8, lp);
      }
    };
    // O^T += V^T P^T over keys 32 c ..: lane group g's k slots are keys 32 c + 4 g + (0..3) and
    // 32 c + 16 + 4 g + (0..3), transposed reads give V's column 16 t + l16 of those.
    auto pv = [&](int c, auto CLEAN) {
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        u32x4 av;
        const char* p = vt + vat[t & 3] + 64 * VX * (t >> 2) + 32 / RPB * VBLK * c;
        if constexpr (E8) {
          const u32x2 v = ds_read_tr8(p);
          av = widen8<false>(v[0], v[1]);
        } else {
          const u32x2 v0 = ds_read_tr((const uint16_t*)p), v1 = ds_read_tr((const uint16_t*)(p + 16 / RPB * VBLK));
          av = (u32x4){v0[0], v0[1], v1[0], v1[1]};
        }
        if constexpr (decltype(CLEAN)::value)
          av = (u32x4){finite_pair<PF16>(av[0]), finite_pair<PF16>(av[1]), finite_pair<PF16>(av[2]), finite_pair<PF16>(av[3])};
        const bf16x8 af = __builtin_bit_cast(bf16x8, av);
#pragma unroll
        for (int gq = 0; gq < PT_NG; ++gq) {
          o[gq][t] = mfma16<PF16>(af, bh[c][gq], o[gq][t]);
          o[gq][t] = mfma16<PF16>(af, bl[c][gq], o[gq][t]);
        }
      }
    };
    // The first reads of a phase go out together; each later one while the MFMAs of an earlier one run.
    constexpr int KR = E8 ? 2 * KS : 4 * KS, KM = 4 * KS * PT_NG / KR;   // K reads, MFMAs of each
    constexpr int VR = E8 ? 1 : 2;                                       // V reads of a fragment
    constexpr int KV = (E8 ? 136 : 48) / KR, VV = (E8 ? 104 : 48) / DT;  // vector instructions beside each
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (next) {
      qk(kb, sn);
    }
    probs(0);
    if constexpr (next) {
      __builtin_amdgcn_sched_group_barrier(0x100, PT_AHEAD, 0);
#pragma unroll
      for (int x = 0; x < KR; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x002, KV, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, KM, 0);
        if (x + PT_AHEAD < KR) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!next) {
      if (__builtin_expect(clean, 0)) {
        probs(1);
        asm volatile("" : "+v"(lsum[0]), "+v"(lsum[1]));  // summed here: P is not kept in registers until after the loop below
        pv(0, std::true_type{});
        pv(1, std::true_type{});
        add_odd_values<PF16, E8, DT, PT_NG>(
            [&](int key, int d) { return vt + key / RPB * VBLK + key % RPB * RB + 16 * ((d * EB / 16) ^ (VX * swz<RB>(key))) + (d * EB) % 16; },
            k0, odds, g, pos, o);
        return;
      }
    }
    pv(0, std::false_type{});
    probs(1);
    __builtin_amdgcn_sched_group_barrier(0x100, VR * PT_AHEAD, 1);
#pragma unroll
    for (int x = 0; x < DT; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x002, VV, 1);
      __builtin_amdgcn_sched_group_barrier(0x008, PT_NG * 2, 1);
      if (x + PT_AHEAD < DT) __builtin_amdgcn_sched_group_barrier(0x100, VR, 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    pv(1, std::false_type{});
    if constexpr (next) {
      scale_s(n + 1, sn);
      top_of(sn, tmax);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, VR * PT_AHEAD, 2);
#pragma unroll
    for (int x = 0; x < DT; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x002, (next ? 32 : 0) / DT, 2);
      __builtin_amdgcn_sched_group_barrier(0x008, PT_NG * 2, 2);
      if (x + PT_AHEAD < DT) __builtin_amdgcn_sched_group_barrier(0x100, VR, 2);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // Tiles t0 .. tfull - 1 lie wholly before all rows of the workgroup: they overlap with the next one's S.  The
  // last few, which are masked, do not.
  const int tfull = min(t1, (rtile.pos(0) + 1) / PT_K);
  int n = t0;
  if (n < t1) {
    pg.place(a, kvh, 64 * win, rend, lane, bad);
    pgn.place(a, kvh, 64 * (win + 1), rend, lane, bad);
    load_k(n, Kb0);
    load_v(n, Vb0);
    if (n + 1 < t1) load_k(n + 1, Kb1);
  }
  // A whole tile with K and V in buffers k0 / v0, the next in k1 / v1.  At its top K(n + 1) and V(n) have landed,
  // and every wave is done with K(n) and V(n - 1).
  float tmax[PT_NG];
  auto whole = [&](auto ROWS, char* k0, char* v0, char* k1, char* v1, f32x4 (*st)[4], f32x4 (*sn)[4]) {
    landed();
    if (n + 1 < t1) load_v(n + 1, v1);
    if (n + 2 < t1) load_k(n + 2, k0);
    if constexpr (decltype(ROWS)::value) tile(std::true_type{}, n, v0, k1, st, sn, tmax);
    ++n;
  };
  // A tile that is masked, or beyond the rows of some waves: its S comes first, so that K is loaded one tile ahead
  // only (kin: K(n + 1) is on its way already).
  auto part = [&](char* k0, char* v0, char* k1, char* v1, bool kin) {
    landed();
    if (n + 1 < t1) {
      if (!kin) load_k(n + 1, k1);
      load_v(n + 1, v1);
    }
    if (PT_K * n <= wlast) {  // else every key of the tile is after the wave's rows
      f32x4 st[PT_NG][4];
      qk(k0, st);
      tile(std::false_type{}, n, v0, k0, st, st, tmax);
    }
    ++n;
  };
  // A wave without rows only loads its part of the tiles (32 sequences of up to 4096 keys, 8 new tokens each, 40
  // query heads to 8: 84 us, where it worked on for nothing 91; from an 8-bit cache 103 and 110).
  auto wholes = [&](auto ROWS) {
    f32x4 sa[PT_NG][4], sb[PT_NG][4];
    landed();
    if constexpr (decltype(ROWS)::value) {
      qk(Kb0, sa);
      scale_s(n, sa);
      top_of(sa, tmax);
    }
    for (;;) {
      whole(ROWS, Kb0, Vb0, Kb1, Vb1, sa, sb);
      if (n >= tfull) break;
      whole(ROWS, Kb1, Vb1, Kb0, Vb0, sb, sa);
      if (n >= tfull) break;
    }
  };
  if (n < tfull) {
    if (wr0 < rtile.nrows) wholes(std::true_type{});
    else wholes(std::false_type{});
  }
  bool kin = true;
  if (n < t1 && ((n - t0) & 1)) {
    part(Kb1, Vb1, Kb0, Vb0, true);
    kin = false;
  }
  while (n < t1) {
    part(Kb0, Vb0, Kb1, Vb1, kin);
    kin = false;
    if (n < t1) part(Kb1, Vb1, Kb0, Vb0, false);
  }

#pragma unroll
  for (int off = 32; off > 0; off >>= 1) bad = min(bad, __shfl_xor(bad, off, 64));
  if (lane == 0) bads[wave] = bad;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PG_W; ++i) bad = min(bad, bads[i]);
  if (bad < kv_cap(a.kv) && tid == 0 && a.kv.bad_flag) *a.kv.bad_flag = 1;
  // The rows: normalised, 16 at a time through a buffer of the wave, so that a store covers whole rows; or a
  // split's unnormalised sums.
  uint16_t* const ow = (uint16_t*)(wave == 0 ? Kb0 : wave == 1 ? Kb1 : wave == 2 ? Vb0 : Vb1);
#pragma unroll
  for (int gq = 0; gq < PT_NG; ++gq) {
    float l = lsum[gq] + __shfl_xor(lsum[gq], 16, 64);
    l = (l + __shfl_xor(l, 32, 64)) * PULL;
    const int row = wr0 + 16 * gq + l16;
    if (nsp > 1) {
      if (row >= rtile.nrows) continue;
      // relative to the maximum itself, without b's rounding
      const float f = raw || mrow[gq] == PG_LOW ? 1.f : __builtin_amdgcn_exp2f(SHIFT - fmaf(mrow[gq], a.scale_log2, brow[gq]));
      l *= f;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[gq][t] *= f;
      const size_t at = ((((size_t)s * a.kv.kv_heads + kvh) * a.tiles + rt) * a.nsplit + split) * a.prows + row;
#pragma unroll
      for (int t = 0; t < DT; ++t) *(f32x4*)&a.part[at * DH + 16 * t + 4 * g] = o[gq][t];
      if (g == 0) a.stat[at] = make_float2(mrow[gq], pos[gq] >= bad ? __builtin_nanf("") : l);
      continue;
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = row_result(o[gq][t][e], inv, pos[gq], bad);
      store4<F16>(&ow[l16 * OROW + 16 * t + 4 * g], y);
    }
    constexpr int C8 = DH / 8;
#pragma unroll
    for (int x = lane; x < 16 * C8; x += 64) {
      const int i = wr0 + 16 * gq + x / C8, c = x % C8;
      const u32x4 v = *(const u32x4*)&ow[(x / C8) * OROW + 8 * c];
      if (i < rtile.nrows)
        *(u32x4*)((uint16_t*)a.O + (size_t)(rtile.sp.r0 + rtile.tok(i)) * a.ldo + (size_t)(kvh * a.group + rtile.head(i)) * DH + 8 * c) = v;
    }
  }
}

// ---------------------------------------------------------------- splits
// Joins the splits of a row: O = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i.  TPR teams of DH / 4 lanes share a
// row and take its splits in turn: one team where a workgroup has rows enough, all of them for many splits
// of few rows.
template <bool F16, int DH, int TPR>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  constexpr int D4 = DH / 4, TEAMS = 256 / D4, RPW = TEAMS / TPR;
  __shared__ f32x4 acc[TPR > 1 ? TEAMS : 1][D4];
  __shared__ float2 st[TPR > 1 ? TEAMS : 1];
  const int per = (a.prows + RPW - 1) / RPW;  // workgroups of a row tile
  const int team = threadIdx.x / D4, lane = threadIdx.x % D4, d = 4 * lane;
  int w = blockIdx.x;
  const int row = (w % per) * RPW + team / TPR;
  w /= per;
  const int rt = w % a.tiles;
  w /= a.tiles;
  const int kvh = w % a.kv.kv_heads, s = w / a.kv.kv_heads;
  const RowTile rtile = row_tile(a, kv_span(a.kv, s), rt);
  const int nsp = splits_of(a, rtile.kend);
  if (nsp == 1) return;  // written already
  const bool mine = row < rtile.nrows;
  if (TPR == 1 && !mine) return;
  const size_t base = (((size_t)s * a.kv.kv_heads + kvh) * a.tiles + rt) * a.nsplit;
  float m = PG_LOW, l = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i = team % TPR; i < nsp && mine; i += TPR) {
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
  if constexpr (TPR > 1) {
    acc[team][lane] = y;
    if (lane == 0) st[team] = make_float2(m, l);
    __syncthreads();
    if (team % TPR || !mine) return;
    m = PG_LOW;
#pragma unroll
    for (int i = 0; i < TPR; ++i) m = fmaxf(m, st[team + i].x);
    l = 0.f;
    y = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < TPR; ++i) {
      const float f = __builtin_amdgcn_exp2f((st[team + i].x - m) * a.scale_log2);
      const f32x4 v = acc[team + i][lane];
      l += f * st[team + i].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += f * v[e];
    }
  }
  const int p = rtile.pos(row);
  const float inv = 1.f / l;
  float o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = row_result(y[e], inv, p, 0x7fffffff);
  store4<F16>((uint16_t*)a.O + (size_t)(rtile.sp.r0 + rtile.tok(row)) * a.ldo + (size_t)(kvh * a.group + rtile.head(row)) * DH + d, o);
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
  a.inv_group = a.group > 1 ? (uint32_t)((1ull << 32) / (unsigned)a.group) + 1 : 0;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)kv.dh);
  const long long all_rows = (long long)kv.max_q * a.group, seqs = (long long)kv.nseq * kv.kv_heads;
  if (all_rows > 0x7fffffffLL - 4096 || seqs > 0x7fffffffLL) {  // what follows of them stays within 64 bits
    zo_set_error("paged_attention: max_q x heads / kv_heads = %lld or nseq x kv_heads = %lld too many", all_rows, seqs);
    return ZO_ERR_UNSUPPORTED;
  }
  // Few rows of a sequence and key head read its keys and little else; more share staged tiles.  With 20 rows (40 heads
  // to 8 of 128), 61 sequences of up to 8192 keys took 209 us here where staged tiles took 220, in 8 bits 124 and 190
  // (heads of 64: 115 and 122, 80 and 134); 16 sequences of up to 1000 keys 22 and 34, in 8 bits 22 and 40.
  const bool many = all_rows > 32;
  const int ng = many || all_rows > 16 ? 2 : 1;
  a.rt_rows = many ? PT_Q : 16 * ng;
  a.prows = (int)(all_rows < a.rt_rows ? all_rows : a.rt_rows);
  const long long tiles = (all_rows + a.rt_rows - 1) / a.rt_rows;
  const long long units = seqs * tiles;
  const long long keys = (long long)kv.max_pages << kv.log2ps;
  // Splits: as many as give 512 workgroups, two per CU (at least that where a split's rows are few), but 64 at most: with
  // three key heads and more 64 fill the CUs, and with one or two more of them gained only for the longest of
  // contexts (one token, 64 and 128 splits: two key heads, 32768 keys 16.3 and 17.3 us, 131072 keys 31.8 and 31.5; four,
  // 30 and 32, 48.5 and 51 us at 65536 and 131072; one key head 15.1 and 15.2, 31 and 24; with 256 and 512 no better).
  // With 128 units or more a split has 2048 keys at least, for
  // it costs a partial result (32 sequences of 2000 keys, 8 key heads: 51 us, in halves 55); with fewer, 256, but
  // up to 512 keys stay whole (300 keys of one sequence: 7.8 us, in halves and a second launch 9.3).
  a.min_keys = units < 128 ? 256 : 2048;
  const long long most = keys <= 512 ? 1 : (keys + a.min_keys - 1) / a.min_keys;
  long long split = ((many && tiles > 1 ? 0 : units - 1) + 512) / units;
  if (split > 64) split = 64;
  if (split > most) split = most;
  if (split < 1) split = 1;
  if (units * split > 0x7fffffffLL) {
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
  const dim3 grid = kv_grid(units * split), block(64 * PG_W);
  a.wgs = (unsigned)(units * split);
  const bool f16 = kv.dtype == ZO_F16;
#define ZO_ROWS(F, E, D)                                                                                    \
  if (many) hipLaunchKernelGGL((k_paged_tile<F, E, D>), grid, block, 0, stream, a);                        \
  else if (ng == 2) hipLaunchKernelGGL((k_paged_rows<F, E, D, 2>), grid, block, 0, stream, a);             \
  else hipLaunchKernelGGL((k_paged_rows<F, E, D, 1>), grid, block, 0, stream, a)
#define ZO_ROWS_D(F, E) \
  if (kv.dh == 64) { ZO_ROWS(F, E, 64); } \
  else { ZO_ROWS(F, E, 128); }
  if (kv.e8) {
    if (f16) { ZO_ROWS_D(true, true); } else { ZO_ROWS_D(false, true); }
  } else {
    if (f16) { ZO_ROWS_D(true, false); } else { ZO_ROWS_D(false, false); }
  }
#undef ZO_ROWS_D
#undef ZO_ROWS
  int st = zo_hip_status(hipGetLastError(), many ? "k_paged_tile" : "k_paged_rows");
  if (st != ZO_OK || split == 1) return st;
  // One team of lanes per row, but for many splits of few rows.
  const int teams = 256 / (kv.dh / 4);
  const bool wide = split > 4 && units * a.prows <= 4096;
  const dim3 jgrid((unsigned)(units * (wide ? a.prows : (a.prows + teams - 1) / teams)));  // at most 511 units here
#define ZO_JOIN(F, D)                                                                                       \
  if (wide) hipLaunchKernelGGL((k_paged_join<F, D, 256 / (D / 4)>), jgrid, dim3(256), 0, stream, a);       \
  else hipLaunchKernelGGL((k_paged_join<F, D, 1>), jgrid, dim3(256), 0, stream, a)
  if (kv.dh == 64) {
    if (f16) { ZO_JOIN(true, 64); } else { ZO_JOIN(false, 64); }
  } else {
    if (f16) { ZO_JOIN(true, 128); } else { ZO_JOIN(false, 128); }
  }
#undef ZO_JOIN
  return zo_hip_status(hipGetLastError(), "k_paged_join");
}
