// Attention of bfloat16 queries over an 8-bit cache (head dim 72): queries of
// one (chain, head) against the first key_len keys of the chain, key ranges
// (splits) joined by a second kernel.
//
// The matrix work is that of the bfloat16 self-attention (rc_attn4.hip):
// scores transposed (S^T = K Q^T), so a lane owns one query and its
// probabilities are in registers the B operand of O^T = V^T P^T; two blocks of
// 32 dims and one of 16 that holds dims 64..71 and the denominator (a row of
// ones behind the values, which sums the rounded probabilities).  e4m3 times a
// power of two is exact in bfloat16, so the 8-bit cache costs no precision
// beyond its own, and the probabilities' rounding to bfloat16 (2^-9 relative
// each, averaged by the sum) is the only one before the result's.
// * Tiles of 64 keys and values (9 KB) go global -> LDS by direct copies into a
//   ring of six; fragments are read as 8-bit values (half of the LDS traffic
//   that bounds the bfloat16 kernel at QH = 1) and converted in registers, once
//   for QH 32x32 units.  (Tiles made bfloat16 in LDS once per workgroup take 18
//   conversions per wave instead of 80, but three passes through LDS: 5 % slower
//   for 723 queries of 4096 keys, no faster for 16384 of 16384.)
// * Of the ring only half a tile's time hides a copy: the register of scale
//   bytes, loaded anew every 64 tiles, is read at the start of each, and the
//   compiler's wait for it, in a loop whose copies it does not know of, is one
//   for all of them.
// * A partial last tile: keys and values behind the last become zeros in LDS,
//   and dim 72 of those keys, which meets +-1 in the queries, is -3.4e38, so
//   that no other place knows about masks.
// * Probabilities are exp2(scale s - m), one fma and one exponential, relative
//   to m = 0 at first: bfloat16 probabilities and float32 sums keep their
//   relative precision over the whole exponent range.  A workgroup one of whose
//   denominators is not inside [2^-40, 2^80] (or is NaN), or one of whose sums
//   of values is not finite, starts again relative to each query's maximum plus
//   24 (probabilities of at most 2^-24).  Logits above 55 lead there, or a query
//   whose logits are all below -28: where every workgroup does, 723 queries of
//   4096 keys take 58 us instead of 33, 16384 of 16384 2860 instead of 1170.
#include "rc_common.h"
#include "rc_launch.h"
#include "rc_quant.h"

#include <algorithm>
#include <cmath>

namespace rc {

// Probabilities relative to a maximum are at most 2^-24, so that the sum of up
// to 2^24 values stays finite wherever their weighted mean does.
constexpr float kHeadroom = 24.0f;

__device__ __forceinline__ int key_perm8(int m) {
  return ((m >> 4) & 1) * 16 + ((m >> 2) & 1) * 8 + ((m >> 3) & 1) * 4 + (m & 3);
}
template <int N> __device__ __forceinline__ void wait_vm8() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// Workgroup barrier with this wave's LDS writes done and its copies in flight.
__device__ __forceinline__ void lds_barrier8() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// This workgroup's chain, head, key range and query rows q0 .. (at most bq, up
// to r1); false if it has none.  Heads and key ranges are shared out to the
// XCDs, so that each has a part of every chain, however ragged the chains' rows
// and keys are, and the query tiles that read the same keys are on one XCD.
// Within an XCD the query tiles are outermost, so that a long chain's are on
// different CUs.  (Six chains of 0..655 rows and 0..4096 keys in a graph 44 us; heads
// outermost 54, a busy tile on every eighth CU; chains outermost 109.)
// The grid holds the query tiles of all chains, or for more chains than the
// arguments hold the longest one's for each.
__device__ __forceinline__ bool locate(const QAttnArgs &a, int bq, int &b, int &h, int &split, int &q0, int &r1) {
  const int n_hs = a.c.heads * a.splits, tiles_q = gridDim.x / n_hs;
  int hy, qt;
  if ((n_hs & 7) == 0) {  // an XCD's share in order of query tiles
    const int x = blockIdx.x & 7, i = blockIdx.x >> 3, per = n_hs >> 3;
    qt = i / per;
    hy = x * per + i - qt * per;
  } else {
    const int L = xcd_logical_id(blockIdx.x, gridDim.x);
    hy = L / tiles_q;
    qt = L - hy * tiles_q;
  }
  h = hy % a.c.heads;
  split = hy / a.c.heads;
  b = 0;
  if (a.chains <= kQArgChains) {
    for (; b < a.chains - 1; ++b) {
      const int nt = (a.rows.arg[b + 1] - a.rows.arg[b] + bq - 1) / bq;
      if (qt < nt) break;
      qt -= nt;
    }
  } else {
    b = qt / (tiles_q / a.chains);
    qt -= b * (tiles_q / a.chains);
  }
  const int2 rr = chain_rows(a.rows, b);
  q0 = rr.x + qt * bq;
  r1 = rr.y;
  return q0 < r1;
}

// A wave holds QH halves of 32 queries.
template <int QH> __global__ __launch_bounds__(256, 2) void qattn_kernel(QAttnArgs a) {
  constexpr int D = kHeadDim;
  constexpr int RAW = 2 * kQTileBytes, STAGES = 6;
  constexpr int BQ = 128 * QH, WQ = 32 * QH;
  constexpr int CONST_OFF = STAGES * RAW;
  __shared__ __attribute__((aligned(1024))) char lds[CONST_OFF + 64];
  // read in place of value dims 72..79: (1, 0, ...); of key dims 72..79: zeros
  char *ones_chunk = lds + CONST_OFF, *zero_chunk = ones_chunk + 8;
  volatile int *flag = (volatile int *)(lds + CONST_OFF + 32);
  if (threadIdx.x == 0) {
    *(V16 *)ones_chunk = V16{{0x00000038u, 0u, 0u, 0u}};
    *flag = 0;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < 4);
  const int g = lane >> 5, r32 = lane & 31;
  const int heads = a.c.heads;
  int b, h, split, q0, r1;
  if (!locate(a, BQ, b, h, split, q0, r1)) return;
  const int keys = a.key_len ? max(0, min(a.key_len[b], a.c.tokens)) : a.c.tokens;
  const int n_tiles = (keys + kQTokens - 1) / kQTokens;
  const int t_beg = (int)((long long)split * n_tiles / a.splits), t_end = (int)((long long)(split + 1) * n_tiles / a.splits);
  const int n = t_end - t_beg, left = keys - t_beg * kQTokens;  // keys from the range's first on
  const uint8_t *data = a.c.data + b * a.c.chain_stride + ((size_t)h * (a.c.tokens / kQTokens) + t_beg) * RAW;
  const uint16_t *scales = (const uint16_t *)(a.c.scales + b * a.c.scale_chain_stride) + (size_t)h * (a.c.tokens / kQTokens) + t_beg;

  // A tile is nine copies of 1 KB: two per wave, and a quarter of the ninth.
  const unsigned lds0 = lds_address(lds);
  auto issue = [&](const uint8_t *from, int slot, int tile) {
    const uint8_t *p = from + (size_t)tile * RAW + wave * 1024;
    const unsigned to = lds0 + slot * RAW + wave * 1024;
    lds_dma16s(p, lane * 16, to);
    lds_dma16s(p + 4096, lane * 16, to + 4096);
    if (lane < 16) lds_dma16s(p + 8192 - wave * 768, lane * 16, to + 8192 - wave * 768);
  };
  auto wait_tiles = [&](int later) {  // at most `later` younger tiles' copies are in flight
    if (later >= 4) wait_vm8<12>();
    else if (later == 3) wait_vm8<9>();
    else if (later == 2) wait_vm8<6>();
    else if (later == 1) wait_vm8<3>();
    else wait_vm8<0>();
  };
  // the keys and values behind the last key of a partial tile (which has
  // arrived) become zeros; every thread of the workgroup calls it
  auto clear_rest = [&](int slot, int tile) {
    const int rest = left - tile * kQTokens;
    if (rest < kQTokens) {
      for (int c = rest * (D / 8) + tid; c < kQTileBytes / 8; c += 256) {
        *(u32x2 *)(lds + slot * RAW + c * 8) = u32x2{0u, 0u};
        *(u32x2 *)(lds + slot * RAW + kQTileBytes + c * 8) = u32x2{0u, 0u};
      }
      lds_barrier8();
    }
  };
  // scale bytes of 64 tiles, one tile's pair per lane
  int sc = 0;
  auto load_scales = [&](int tile) { sc = scales[min(tile + lane, n - 1)]; };

  bf16x8 qf[QH][5];
#pragma unroll
  for (int hh = 0; hh < QH; ++hh) {
    const bf16 *qrow = a.q + min(q0 + wave * WQ + hh * 32 + r32, r1 - 1) * a.ldq + h * D;
#pragma unroll
    for (int c = 0; c < 5; ++c) {
      const int d0 = c * 16 + g * 8;
      qf[hh][c] = Mfma<bf16>::zero();
      if (d0 < D) qf[hh][c] = *(const bf16x8 *)(qrow + d0);
    }
    if (g) qf[hh][4][0] = (bf16)(a.scale_log2 < 0.0f ? -1.0f : 1.0f);
  }
  auto no_keys = [&]() {
    for (int q = q0 + wave * WQ; q < min(q0 + wave * WQ + WQ, r1); ++q) {
      if (a.splits == 1) {
        if (lane < D / 4) *(u32x2 *)(a.out + q * a.ldo + h * D + lane * 4) = u32x2{0u, 0u};
      } else if (lane == 0) {
        float *ml = a.ml + (((size_t)split * a.total_rows + q) * heads + h) * 2;
        ml[0] = -INFINITY;
        ml[1] = 0.0f;
      }
    }
  };
  if (n == 0) {
    no_keys();
    return;
  }
  // (consumed here so that no wait for them is left inside the tile loop)
#pragma unroll
  for (int hh = 0; hh < QH; ++hh)
#pragma unroll
    for (int c = 0; c < 5; ++c) asm volatile("" : "+v"(qf[hh][c]));

  const int my_key = key_perm8(r32), k_off = my_key * D + g * 8;
  auto kread = [&](const char *t, int st, u32x2 *kr) {
    const char *row = t + st * 32 * D + k_off;
#pragma unroll
    for (int c = 0; c < 4; ++c) kr[c] = *(const u32x2 *)(row + c * 16);
    kr[4] = *(const u32x2 *)(g ? zero_chunk : row + 64);
  };
  // V^T operands by transpose reads: within a 16-lane group, lane j supplies
  // the address of an 8-dim chunk of key j / 2, and lane i receives dim i of
  // the eight keys
  typedef int v2i __attribute__((ext_vector_type(2)));
  const int tw = lane >> 4, tj = lane & 15;
  const int v_off = kQTileBytes + ((tj >> 1) + (tw >> 1) * 8) * D + 16 * (tw & 1) + 8 * (tj & 1);
  const int w_off = kQTileBytes + ((tj >> 1) + (tw & 1) * 16 + (tw >> 1) * 8) * D + 64;
  // k = 0..3: dims 32 (k % 2) .. +31 of keys 16 (k / 2) + 8 g ..; k = 4: dims 64..79 of the 32 keys
  auto vread = [&](const char *t, int st, int k) {
    const char *p = k < 4 ? t + v_off + (st * 32 + (k >> 1) * 16) * D + (k & 1) * 32
                          : (tj & 1) ? ones_chunk : t + w_off + st * 32 * D;
    const v2i v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i *)p);
    return u32x2{(uint32_t)v[0], (uint32_t)v[1]};
  };
  const f32x16 zero16 = {};
  // chunk c of the keys: 16 dims; dim 72 of masked keys (rest: keys from the sub-tile's first on) is -3.4e38
  auto kfrag = [&](const u32x2 *kr, int c, float f, int rest) {
    bf16x8 k = q_bf16x8(kr[c], f);
    if (c == 4 && rest < 32 && g && my_key >= rest) k[0] = __builtin_bit_cast(bf16, (uint16_t)0xFF7F);
    return k;
  };
  const float c1 = a.scale_log2;

  f32x16 o[QH][2];  // dims 0..63
  f32x4 o2[QH][2];  // dims 64..71, the denominator (row 72) and seven unused rows, queries 0..15 and 16..31
  float m_ref[QH];
#pragma unroll
  for (int hh = 0; hh < QH; ++hh) m_ref[hh] = 0.0f;
  bool again = false;
  for (;;) {
    const uint8_t *from = data;
    asm volatile("" : "+s"(from));  // (addresses are made here, not ahead of the outer loop)
    if (again) {
#pragma unroll
      for (int hh = 0; hh < QH; ++hh) m_ref[hh] = -INFINITY;
#pragma nounroll
      for (int i = 0; i < n; ++i) {
        if ((i & 63) == 0) load_scales(i);
        issue(from, 0, i);
        wait_vm8<0>();
        lds_barrier8();
        clear_rest(0, i);
        const float fk = q_factor(__builtin_amdgcn_readlane(sc, i & 63) & 255);
        for (int st = 0; st < 2; ++st) {
          u32x2 kr[5];
          kread(lds, st, kr);
          f32x16 s[QH];
#pragma unroll
          for (int c = 0; c < 5; ++c) {
            const bf16x8 k = kfrag(kr, c, fk, left - i * kQTokens - st * 32);
#pragma unroll
            for (int hh = 0; hh < QH; ++hh)
              s[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[hh][c], c == 0 ? zero16 : s[hh], 0, 0, 0);
          }
#pragma unroll
          for (int hh = 0; hh < QH; ++hh)
#pragma unroll
            for (int e = 0; e < 16; ++e) m_ref[hh] = fmaxf(m_ref[hh], s[hh][e] * c1);
        }
        lds_barrier8();
      }
#pragma unroll
      for (int hh = 0; hh < QH; ++hh) {
        const float m = half_swap_max(m_ref[hh]);
        m_ref[hh] = m == -INFINITY ? 0.0f : m + kHeadroom;
      }
      lds_barrier8();
    }
    load_scales(0);
#pragma nounroll
    for (int i = 0; i < min(n, STAGES - 1); ++i) issue(from, i, i);
    wait_tiles(min(n - 1, STAGES - 2));
    asm volatile("" : "+v"(sc));
    lds_barrier8();
    if (n == 1) clear_rest(0, 0);
#pragma unroll
    for (int hh = 0; hh < QH; ++hh)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        o[hh][t] = zero16;
        o2[hh][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    // A tile is worked off in units of 32 queries x 32 keys, two at a time:
    // the scores of unit 0; the scores of unit 1 with the exponentials of
    // unit 0; PV of unit 0 with the exponentials of unit 1; PV of unit 1.
    // QH = 2: the units are the wave's two query halves on one key sub-tile,
    // whose operands are converted once; QH = 1: the two key sub-tiles.
    constexpr int NK = QH == 2 ? 1 : 2;  // key sub-tiles per pair of units
    u32x2 kr[NK][5];
#pragma unroll
    for (int q = 0; q < NK; ++q) kread(lds, q, kr[q]);
    int slot = 0;
    for (int i = 0; i < n; ++i) {
      const char *t = lds + slot * RAW;
      slot = slot == STAGES - 1 ? 0 : slot + 1;
      if ((i & 63) == 0 && i) load_scales(i);
      const int pair = __builtin_amdgcn_readlane(sc, i & 63), rest = left - i * kQTokens;
      const float fk = q_factor(pair & 255), fv = q_factor(pair >> 8), fw = tj == 8 ? 1.0f : fv;  // (the row of ones)
#pragma unroll
      for (int st = 0; st < 2; st += NK) {
        f32x16 s[2];
        u32x2 vr[NK][5];
        bf16x8 kf[5], vf[5];
        float pe[2][16];
        bf16x8 pf[2][2];
        auto exps = [&](int u, int e0, int e1) {  // pinned to their place between the MFMAs
#pragma unroll
          for (int e = e0; e < e1; ++e) {
            float x = s[u][e];
            asm volatile("" : "+v"(x));
            pe[u][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x, c1, -m_ref[u % QH]));
          }
        };
        auto cvt = [&](int u, int c) {
#pragma unroll
          for (int k = 0; k < 8; ++k) pf[u][c][k] = (bf16)pe[u][c * 8 + k];
        };
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int c = 0; c < 5; ++c) {
            if (u < NK) kf[c] = kfrag(kr[u], c, fk, rest - (st + u) * 32);
            s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], qf[u % QH][c], c == 0 ? zero16 : s[u], 0, 0, 0);
            if (u < NK) vr[u][c] = vread(t, st + u, c);
            if (u == 1 && c > 0) exps(0, 4 * (c - 1), 4 * c);
            __builtin_amdgcn_sched_barrier(0);
          }
        cvt(0, 0);
        cvt(0, 1);
        asm volatile("" : "+v"(pf[0][0]), "+v"(pf[0][1]));  // (not to be moved past the branch)
        if (st + NK == 2 && i + 1 < n) {
          wait_tiles(min(n - 2 - i, STAGES - 3));  // tile i + 1 has arrived
          lds_barrier8();
          if (i + STAGES - 1 < n) issue(from, slot < 2 ? slot + STAGES - 2 : slot - 2, i + STAGES - 1);
          if (i + 2 == n) clear_rest(slot, i + 1);
        }
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int hh = u % QH;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (u < NK) vf[k] = q_bf16x8(vr[u][k], fv);
            o[hh][k & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k], pf[u][k >> 1], o[hh][k & 1], 0, 0, 0);
            if (u == 0) exps(1, 3 * k, 3 * k + 3);
            if (u == 0 && k == 3) cvt(1, 0);
            if (u == 1 && k == 0 && (st + NK < 2 || i + 1 < n)) {
#pragma unroll
              for (int q = 0; q < NK; ++q)
                kread(st + NK < 2 ? t : lds + slot * RAW, st + NK < 2 ? st + NK + q : q, kr[q]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          // dims 64..79: the probabilities of queries 0..15 and 16..31 as
          // operands of 32 keys (rows of 16 lanes exchanged between the two)
          if (u < NK) vf[4] = q_bf16x8(vr[u][4], fw);
          bf16x8 pq[2];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const auto r = __builtin_amdgcn_permlane16_swap(((const unsigned *)&pf[u][0])[w], ((const unsigned *)&pf[u][1])[w],
                                                            false, false);
            ((unsigned *)&pq[0])[w] = r[0];
            ((unsigned *)&pq[1])[w] = r[1];
          }
#pragma unroll
          for (int q = 0; q < 2; ++q)
            o2[hh][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[4], pq[q], o2[hh][q], 0, 0, 0);
          if (u == 0) {
            exps(1, 12, 16);
            cvt(1, 1);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (again) break;
    bool bad = false;
    float nan0 = 0.0f;  // 0, or NaN if a sum is not finite
#pragma unroll
    for (int hh = 0; hh < QH; ++hh)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        bad = bad || (tw == 2 && !(o2[hh][q][0] < 0x1p80f && o2[hh][q][0] > 0x1p-40f));
#pragma unroll
        for (int e = 0; e < 16; ++e) nan0 = __builtin_fmaf(o[hh][q][e], 0.0f, nan0);
#pragma unroll
        for (int e = 0; e < 4; ++e) nan0 = __builtin_fmaf(o2[hh][q][e], 0.0f, nan0);
      }
    if (__any(bad || nan0 != 0.0f) && lane == 0) *flag = 1;
    __syncthreads();
    if (!*flag) break;
    again = true;
  }

#pragma unroll
  for (int hh = 0; hh < QH; ++hh) {
    // the denominators: row 72 is row 8 of the last block, lanes 32..47
    const float l0 = __shfl(o2[hh][0][0], 32 + tj, 64), l1 = __shfl(o2[hh][1][0], 32 + tj, 64);
    const float l_tot = (r32 >> 4) ? l1 : l0;
    const int q_base = q0 + wave * WQ + hh * 32, my_q = q_base + r32;
    auto put = [&](int q, int d, const f32x4 v, float den) {
      if (a.splits == 1) {
        const float inv = den == 0.0f ? 0.0f : 1.0f / den;  // (0: every score is -infinity)
        *(bf16x4 *)(a.out + q * a.ldo + h * D + d) =
            bf16x4{(bf16)(v[0] * inv), (bf16)(v[1] * inv), (bf16)(v[2] * inv), (bf16)(v[3] * inv)};
      } else {
        *(f32x4 *)(a.part + ((size_t)split * a.total_rows + q) * heads * D + h * D + d) = v;
      }
    };
    if (my_q < r1) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          put(my_q, t * 32 + i * 8 + g * 4,
              f32x4{o[hh][t][i * 4], o[hh][t][i * 4 + 1], o[hh][t][i * 4 + 2], o[hh][t][i * 4 + 3]}, l_tot);
    }
    if (tw < 2) {
      if (q_base + tj < r1) put(q_base + tj, 64 + tw * 4, o2[hh][0], l0);
      if (q_base + 16 + tj < r1) put(q_base + 16 + tj, 64 + tw * 4, o2[hh][1], l1);
    }
    if (a.splits > 1 && g == 0 && my_q < r1) {
      float *ml = a.ml + (((size_t)split * a.total_rows + my_q) * heads + h) * 2;
      ml[0] = l_tot == 0.0f ? -INFINITY : m_ref[hh];  // (a range whose scores are all -infinity counts as one without keys)
      ml[1] = l_tot;
    }
  }
}

// Few queries (at most 16 of a chain per workgroup): bound by the cache's
// bytes, so each of eight waves streams tiles of its own (every eighth of the
// key range) through a ring of two without a barrier, with a running maximum,
// and the waves' results are joined in LDS.  (The ring is drained at each tile:
// the wait for the scale bytes, as above.  Two workgroups of four waves on a
// CU need twice the key splits: 64 queries of 4096 keys and 33 of 16384 took 5
// and 7 % longer.)  One query of 16384 keys: 14.5 us with its combine, 38 MB or
// 7.4 us of the cache; 11 splits, in which a wave takes two or three tiles, then
// the ends and the second launch.  16x16x32 blocks: rows m of two 16-key
// operands are keys (m>>2)*8 + (m&3) and those + 4 of 32, so that a lane's
// eight scores are those of the eight keys that PV takes from it.
constexpr int kFewWaves = 8;
__global__ __launch_bounds__(64 * kFewWaves, 2) void qattn_few_kernel(QAttnArgs a) {
  constexpr int D = kHeadDim, RAW = 2 * kQTileBytes, STAGES = 2, W = kFewWaves;
  __shared__ __attribute__((aligned(1024))) char lds[W * STAGES * RAW + 64];
  __shared__ float wave_m[W][16], wave_l[W][16];
  char *ones_chunk = lds + W * STAGES * RAW;  // read in place of value dims 72..79
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < W);
  const int l16 = lane & 15, lq = lane >> 4, heads = a.c.heads;
  int b, h, split, q0, r1;
  if (!locate(a, 16, b, h, split, q0, r1)) return;
  const int keys = a.key_len ? max(0, min(a.key_len[b], a.c.tokens)) : a.c.tokens;
  const int n_tiles = (keys + kQTokens - 1) / kQTokens;
  const int t_beg = (int)((long long)split * n_tiles / a.splits) + wave;
  const int t_end = (int)((long long)(split + 1) * n_tiles / a.splits);
  const int n = t_beg < t_end ? (t_end - t_beg + W - 1) / W : 0;  // tiles t_beg + W i
  const uint8_t *data = a.c.data + b * a.c.chain_stride + ((size_t)h * (a.c.tokens / kQTokens) + t_beg) * RAW;
  const uint16_t *scales = (const uint16_t *)(a.c.scales + b * a.c.scale_chain_stride) + (size_t)h * (a.c.tokens / kQTokens) + t_beg;
  char *ring = lds + wave * STAGES * RAW;
  const unsigned ring0 = lds_address(ring);
  auto issue = [&](int slot, int i) {
    const uint8_t *p = data + (size_t)i * W * RAW;
#pragma unroll
    for (int c = 0; c < RAW / 1024; ++c) lds_dma16s(p + c * 1024, lane * 16, ring0 + slot * RAW + c * 1024);
  };
  if (tid == 0) *(V16 *)ones_chunk = V16{{0x00000038u, 0u, 0u, 0u}};
  int sc = 0;  // scale bytes of 64 of the wave's tiles, one pair per lane
  if (n > 0) sc = scales[W * min(lane, n - 1)];
  bf16x8 qf[3];
  const bf16 *qrow = a.q + min(q0 + l16, r1 - 1) * a.ldq + h * D;
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    qf[c] = Mfma<bf16>::zero();
    if (c < 2 || lq == 0) qf[c] = *(const bf16x8 *)(qrow + c * 32 + lq * 8);
  }
  for (int i = 0; i < min(n, STAGES); ++i) issue(i, i);
  __syncthreads();  // (the ones)
  const f32x4 zero4 = {0.0f, 0.0f, 0.0f, 0.0f};
  f32x4 o[5];  // dims 16 d + 4 lq + e (72: the denominator) of query l16
#pragma unroll
  for (int d = 0; d < 5; ++d) o[d] = zero4;
  float ref = -INFINITY;  // the running maximum + kHeadroom
  typedef int v2i __attribute__((ext_vector_type(2)));
  const int k_off = ((l16 >> 2) * 8 + (l16 & 3)) * D + lq * 8;
  const int v_off = kQTileBytes + (lq * 8 + (l16 >> 1)) * D + 8 * (l16 & 1);
  int slot = 0;
  for (int i = 0; i < n; ++i) {
    if (i + 1 < n) wait_vm8<9>();
    else wait_vm8<0>();
    char *tile = ring + slot * RAW;
    const int left = keys - (t_beg + W * i) * kQTokens;
    if (left < kQTokens) {  // keys and values behind the last become zeros
      for (int c = left * (D / 8) + lane; c < kQTileBytes / 8; c += 64) {
        *(u32x2 *)(tile + c * 8) = u32x2{0u, 0u};
        *(u32x2 *)(tile + kQTileBytes + c * 8) = u32x2{0u, 0u};
      }
    }
    const int pair = __builtin_amdgcn_readlane(sc, i & 63);
    const float fk = q_factor(pair & 255), fv = q_factor(pair >> 8), fw = l16 == 8 ? 1.0f : fv;  // (the row of ones)
    f32x4 s[4];  // keys 32 (t / 2) + 8 lq + 4 (t % 2) + e
    float m = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char *krow = tile + k_off + ((t >> 1) * 32 + (t & 1) * 4) * D;
#pragma unroll
      for (int c = 0; c < 3; ++c) {
        u32x2 raw = {0u, 0u};
        if (c < 2 || lq == 0) raw = *(const u32x2 *)(krow + c * 32);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q_bf16x8(raw, fk), qf[c], c == 0 ? zero4 : s[t], 0, 0, 0);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] *= a.scale_log2;
        if (left < kQTokens && (t >> 1) * 32 + lq * 8 + (t & 1) * 4 + e >= left) s[t][e] = -INFINITY;
        m = fmaxf(m, s[t][e]);
      }
    const auto other = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = half_swap_max(fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1])));
    m = fmaxf(m + kHeadroom, ref);
    const float m0 = m == -INFINITY ? 0.0f : m, f = __builtin_amdgcn_exp2f(ref - m0);
    ref = m;
    bf16x8 pf[2];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) pf[t >> 1][(t & 1) * 4 + e] = (bf16)__builtin_amdgcn_exp2f(s[t][e] - m0);
#pragma unroll
    for (int d = 0; d < 5; ++d) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[d][e] *= f;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const char *p = d == 4 && (l16 & 1) ? ones_chunk : tile + v_off + c * 32 * D + d * 16;
        const v2i raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i *)p);
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q_bf16x8(u32x2{(uint32_t)raw[0], (uint32_t)raw[1]}, d == 4 ? fw : fv),
                                                       pf[c], o[d], 0, 0, 0);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
    if (i + STAGES < n) issue(slot, i + STAGES);
    slot ^= 1;
    if (((i + 1) & 63) == 0 && i + 1 < n) sc = scales[W * min(i + 1 + lane, n - 1)];
  }
  // joined: query r's dims of wave w at lds + (w * 16 + r) * 76 floats
  constexpr int LD = D + 4;
  __syncthreads();
  float *res = (float *)lds;
#pragma unroll
  for (int d = 0; d < 5; ++d)
    if (d < 4 || lq < 2) *(f32x4 *)(res + (wave * 16 + l16) * LD + d * 16 + lq * 4) = o[d];
  if (lq == 2) {  // dim 72 is row 8 of the last block
    wave_m[wave][l16] = ref;
    wave_l[wave][l16] = o[4][0];
  }
  __syncthreads();
  const int nq = min(16, r1 - q0);
  for (int c = tid; c < nq * (D / 4); c += 64 * W) {
    const int q = c / (D / 4), dim = (c - q * (D / 4)) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, wave_m[w][q]);
    f32x4 num = zero4;
    float den = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = M == -INFINITY ? 1.0f : exp2f(wave_m[w][q] - M);  // (no maximum: sums are 0, or NaN)
      const f32x4 v = *(const f32x4 *)(res + (w * 16 + q) * LD + dim);
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += f * v[e];
      den += f * wave_l[w][q];
    }
    if (a.splits == 1) {
      const float inv = den == 0.0f ? 0.0f : 1.0f / den;
      *(bf16x4 *)(a.out + (q0 + q) * a.ldo + h * D + dim) =
          bf16x4{(bf16)(num[0] * inv), (bf16)(num[1] * inv), (bf16)(num[2] * inv), (bf16)(num[3] * inv)};
    } else {
      *(f32x4 *)(a.part + ((size_t)split * a.total_rows + q0 + q) * heads * D + h * D + dim) = num;
      if (dim == 0) {
        float *ml = a.ml + (((size_t)split * a.total_rows + q0 + q) * heads + h) * 2;
        ml[0] = M == -INFINITY && den != 0.0f ? 0.0f : M;  // (NaN: kept by the combine)
        ml[1] = den;
      }
    }
  }
}

// O = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m), in split order, over
// the ranges that hold keys (m_s is -inf for the others); a row without keys
// is 0.  One thread per (row, head, 4 dims).
__global__ __launch_bounds__(64) void qattn_combine_kernel(QAttnArgs a) {
  constexpr int G = kHeadDim / 4;
  const int heads = a.c.heads, C = heads * kHeadDim;
  const long long i = (long long)blockIdx.x * 64 + threadIdx.x;
  if (i >= (long long)a.total_rows * heads * G) return;
  const int r = (int)(i / (heads * G)), rem = (int)(i - (long long)r * heads * G), h = rem / G, d = (rem - h * G) * 4;
  float2 ml[kQMaxSplits];
  f32x4 p[kQMaxSplits];
#pragma unroll
  for (int s = 0; s < kQMaxSplits; ++s)
    if (s < a.splits) {
      ml[s] = *(const float2 *)(a.ml + (((size_t)s * a.total_rows + r) * heads + h) * 2);
      p[s] = *(const f32x4 *)(a.part + ((size_t)s * a.total_rows + r) * C + h * kHeadDim + d);
    }
  float M = -INFINITY;
#pragma unroll
  for (int s = 0; s < kQMaxSplits; ++s)
    if (s < a.splits) M = fmaxf(M, ml[s].x);
  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  float den = 0.0f;
#pragma unroll
  for (int s = 0; s < kQMaxSplits; ++s)
    if (s < a.splits && ml[s].x != -INFINITY) {
      const float w = exp2f(ml[s].x - M - 4.0f);  // (sixteen sums that are finite stay so together)
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += w * p[s][e];
      den += w * ml[s].y;
    }
  const float inv = M == -INFINITY ? 0.0f : 1.0f / den;
  *(bf16x4 *)(a.out + r * a.ldo + h * kHeadDim + d) =
      bf16x4{(bf16)(num[0] * inv), (bf16)(num[1] * inv), (bf16)(num[2] * inv), (bf16)(num[3] * inv)};
}

// Kernel and key splits: the pair with the least estimated time.  A tile of 64
// keys takes a CU's two workgroups 1.45 us at QH = 1 and 2.3 at QH = 2, a lone
// one 0.7 of that; the ends 6 us (8.5 for two) and 8; a combine 4 us and its bytes
// at about 4 TB/s.  Of the kernel for few queries a wave takes a tile in 1.75 us,
// a workgroup's ends take 3, one after the other on a CU (33 queries of 16384 keys
// in 5, 10 and 16 splits 21.1, 24.8 and 27.6), and the cache's bytes at most 5.5
// TB/s.  Best of each with its combine, us in a captured graph (on a stream, where
// a launch overlaps the end of the one before, 2 to 4 less; few, QH = 1, QH = 2):
// one query of 16384 keys 16.4, 26.6, 34.2; one of 4096 10.8, 13.9, 16.1; 64 of
// 4096 13.9, 16.6, 19.2; 154 of 4096 19.4, 23.0, 24.8; 154 of 16384 51, 37.1, 39.4;
// 723 of 4096 QH = 1 37.2 (five splits), QH = 2 38.9; 1639 of 4096 61.4 and 59.1; 4096
// of 4096 95.5 and 100.1; 1639 of 16384 170 and 159; 16384 of 16384 1396 and 1168.
// (The constants hold the drain of the rings.)
QAttnPlan plan_qattention(const int *offsets, int chains, int heads, int tokens) {
  const int n_tiles = tokens / kQTokens;
  const long long rows = offsets ? offsets[chains] : (long long)chains * tokens;
  QAttnPlan best{1, 1, 0};
  double best_us = 1e30;
  for (int qh = 0; qh <= 2; ++qh) {
    const int bq = qh ? 128 * qh : 16;
    long long qtiles = 0, most = 0, full = 0;
    for (int b = 0; b < chains; ++b) {
      const int n = offsets ? offsets[b + 1] - offsets[b] : tokens, t = n / bq + (n % bq != 0);
      qtiles += t;
      most = std::max(most, (long long)t);
      full += n > 0;
    }
    const long long grid = (chains <= kQArgChains ? qtiles : chains * most) * heads;
    for (int sp = 1; sp <= std::min(n_tiles, kQMaxSplits) && (sp == 1 || rows * heads * sp <= kQMaxSplitRows); ++sp) {
      const double wgs = (double)qtiles * heads * sp, tiles = (n_tiles + sp - 1) / sp;
      double us = sp > 1 ? 4.0 + rows * heads * kHeadDim * 4.0 * (sp + 1) / 4e6 : 0.0;
      if (qh == 0)
        us += 2.5 + std::max(std::ceil(wgs / 256) * (3.0 + 1.75 * std::ceil(tiles / kFewWaves)),
                             3.0 + full * heads * (double)tokens * 2 * kHeadDim / 5.5e6);
      else
        us += (qh == 2 ? 8.0 : wgs <= 256 ? 6.0 : 8.5) +
              tiles * (qh == 1 ? 1.45 : 2.3) * (wgs <= 256 ? 0.7 : std::ceil(wgs / 512));
      if (us < best_us) {
        best_us = us;
        best = QAttnPlan{qh, sp, grid * sp};
      }
    }
  }
  return best;
}

hipError_t launch_qattention(const QAttnArgs &args, int chains, const QAttnPlan &p, hipStream_t s) {
  if (p.workgroups <= 0 || args.total_rows <= 0) return hipSuccess;
  if (p.workgroups > kQMaxWorkgroups) return hipErrorInvalidValue;
  QAttnArgs a = args;
  // (a scale of 0 becomes one that rounds away: the masks' -3.4e38 must keep its sign)
  if (std::fabs(a.scale_log2) < 1e-30f) a.scale_log2 = 1e-30f;
  a.chains = chains;
  const dim3 grid((unsigned)p.workgroups);
  if (p.qh == 0) rc_launch(qattn_few_kernel, grid, dim3(64 * kFewWaves), 0, s, a);
  else if (p.qh == 2) rc_launch(qattn_kernel<2>, grid, dim3(256), 0, s, a);
  else rc_launch(qattn_kernel<1>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_qattention_combine(const QAttnArgs &a, hipStream_t s) {
  if (a.total_rows <= 0 || a.splits <= 1) return hipSuccess;
  const long long n = (long long)a.total_rows * a.c.heads * (kHeadDim / 4);
  rc_launch(qattn_combine_kernel, dim3((unsigned)((n + 63) / 64)), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace rc
