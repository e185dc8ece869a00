// Head-group masked attention at decode over the 4-bit KV cache.
//
// The mathematics of attention_decode.hip with K and V read as codes: a row
// stands for low_g + s_g c_d in the dimensions d of group g, so
//   score  = sum_g s_g (c . q)_g + low_g sum(q)_g,
//   output = sum_j p_j s_jg (16 + c_jd) + p_j (low_jg - 16 s_jg).
// Nothing is dequantised.
//
// A wave takes tiles of 32 keys of one (sequence, KV head) pair and all query heads
// of the KV head.  Short contexts: one workgroup per pair, its waves take tiles in
// turn, meet in LDS and store o.  Longer ones: every wave takes an equal run of the
// active pairs' tiles (decode_split.h); or, token-major, a workgroup a run of whole
// rows for eight KV heads.  Both leave a (maximum, sum, unnormalised o) per run, and
// a second kernel joins them.
//
// The MFMAs' sixteen columns (rows, for P.V) are (head h, 32-wide group g of the
// dimensions): 4 heads x 4 groups, 8 x 2 in two sets (groups 0 and 1, 2 and 3) or
// 16 x 1 in four, by the query heads per KV head, so that a scale multiplies a
// value of one group where it stands and no lane repeats another's work.  Per
// tile and set:
//   scores  D[key][h, g] = c . q over group g, one 16x16x128 fp8 MFMA per 16
//           keys: a byte 0000cccc is the e4m3 number c 2^-9, so a mask (and a
//           shift) makes operands of the codes; q as two e4m3 terms (its eight
//           bits, or what of them is above 2^-22 of the head's largest, scaled
//           by a power of two per head that the MFMA's block scale takes back)
//           with zeros outside group g.  The scales s_g[key]
//           come in the same layout from a 16x16x16 bf16 MFMA of the rows'
//           (scale, low) with a one-hot operand, low_g sum(q)_g from one with
//           sum(q) in three bf16 parts (24 bits).  The sets are added, then the
//           groups within the lanes of a head, which share out their four keys;
//   softmax online per head, fp32.  The maximum moves only when a score passes
//           it by 8 (in the exponent), so p <= 2^8, and most tiles rescale
//           nothing;
//   P.V     p s_g [h, g][key] in two bf16 parts (2^-16 relative), two MFMAs for
//           each nibble of the words, with the set of its group; 16 + c is a bf16
//           with exponent 2^4 and the code in its top mantissa bits: a shift and
//           an and-or make two.  Row (h, g) of nibble n counts where g = n mod 4.
// The low terms of P.V are fp32 sums per (head, group) beside it.
//
// Bound by the cache's bytes (32 x 8192 keys, 8 KV heads, groups of 32, head-major:
// 336 MB in 67 us with its join, 5.0 TB/s; 64 ragged ones of up to 32768, groups of
// 64: 1.2 GB in 227, 5.3; a pure read of the same shape 6.1), short calls by latency
// (500 keys: 6.8 us).  A tile is 175 vector instructions; two in flight a wave
// (three or four, or two computed together, cost 1-2 us a call in code and in loads
// past the end).  More query heads per KV head are bound by the sets: each multiplies
// 128 deep with zeros outside its groups and keeps its own q (32 x 8192 keys, 32
// query heads, groups of 32, 64, 128: 8 per KV head 44, 44 and 41 us for bytes that
// a read takes 27, 24 and 23 for; 16 per KV head 48, 35, 34 for 14, 12, 12).  With 16
// and groups of 32 the registers run out: 37 of a lane are spilled (23 in the kernel
// of a workgroup per pair), accesses inside the loop over tiles among them.
#include <algorithm>

#include "common.h"
#include "decode_split.h"
#include "kernels.h"
#include "launch.h"
#include "tile256.h"

namespace wide {
namespace {

constexpr int kTile = 32;   // keys per tile

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 16x16x16 bf16 MFMA.  Lane l holds A[row = l%16][k = (l/16)*4 .. +4] and
// B[col = l%16][k = (l/16)*4 .. +4]; the result is laid out as mfma16's.
__device__ __forceinline__ f32x4 mfma16k16(u32x2 a, u32x2 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0,
                                                   0);
}

// Two codes (nibble N of either half of w, N = 0..3) as the bf16 pair 16 + c.
// The exponents come in a register: an and-or with two literals or two scalars
// is two instructions.
template <int N>
__device__ __forceinline__ uint32_t codes(uint32_t w, uint32_t sixteens) {
  constexpr int S = 4 * N - 3;  // bits the nibble moves down
  return ((S < 0 ? w << (S < 0 ? -S : 0) : w >> (S < 0 ? 0 : S)) & 0x00780078u) | sixteens;
}

// The (scale, low) words of a row as a 16x16x16 operand.  NG = 4: lanes with an
// even l/16 hold the four scales, the others the four lows; NG = 2: (s0, s1,
// low0, low1) in every lane; NG = 1: (s0, low0, 0, 0).
template <int NG>
__device__ __forceinline__ u32x2 load_meta(bufview_t v, uint32_t off, uint32_t soff) {
  if constexpr (NG == 1)
    return u32x2{(uint32_t)__builtin_amdgcn_raw_buffer_load_b32(v, (int)off, (int)soff, 0), 0u};
  else
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(v, (int)off, (int)soff, 0));
}

typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16x16x128 MFMA of e4m3 bytes.  Lane l holds A[row = l%16] and B[col = l%16],
// 32 bytes each of k block l/16 (the same order on both sides); the result is
// laid out as mfma16's.  Codes c stand for c 2^-9 (undone by A's scale);
// b_scale is the exponent byte of this lane's column.
__device__ __forceinline__ f32x4 mfma_codes(i32x8 a, i32x8 b, f32x4 c, int b_scale) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 127 + 9, 0, b_scale);
}

// Lane l ^ D of each quad; lane R of each quad, of each pair of lanes.
template <int D>
__device__ __forceinline__ float quad_xor(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), D == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true));
}
template <int R>
__device__ __forceinline__ float pair_bcast(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), R == 0 ? 0xA0 : 0xF5, 0xF, 0xF, true));
}
template <int R>
__device__ __forceinline__ float quad_bcast(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), R * 0x55, 0xF, 0xF, true));
}

// f(r, p of row r) for the four rows of a lane whose head's GC lanes hold the
// rows r = v GC + (lane of the head).
template <int GC, class F>
__device__ __forceinline__ void head_rows(const float (&p)[4 / GC], F f) {
  if constexpr (GC == 4) {
    f(0, quad_bcast<0>(p[0]));
    f(1, quad_bcast<1>(p[0]));
    f(2, quad_bcast<2>(p[0]));
    f(3, quad_bcast<3>(p[0]));
  } else if constexpr (GC == 2) {
    f(0, pair_bcast<0>(p[0]));
    f(1, pair_bcast<1>(p[0]));
    f(2, pair_bcast<0>(p[1]));
    f(3, pair_bcast<1>(p[1]));
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) f(r, p[r]);
  }
}

template <int NG>
struct Tile {
  u32x4 kc[2];        // lane: key 16t + l%16, words 4 (l/16) .. +4
  u32x2 km[2];        // lane: (scale, low) of that key
  uint32_t vc[2][4];  // lane: key 16t + 4 (l/16) + r, word l%16
  u32x2 vm[2];        // as km
};

// One wave's attention over tiles of one pair.  H (4, 8 or 16) at least the query
// heads per KV head.
template <int NG, int H>
struct Attend {
  static constexpr int GC = 16 / H;    // groups of a set
  static constexpr int NS = H / 4;     // sets
  static constexpr int V = 4 / GC;     // of a 16-key half's scores, those one lane goes on with

  int l16, g4, h, gl;                  // this lane's column: head, group of the set
  u32x4 qr[NS];
  i32x8 q_hi[NS], q_lo[NS];            // q 2^e in two e4m3 terms, the second times 2^5
  int q_sc;                            // the exponent byte that undoes e
  u32x2 b_low[NS][2];                  // sum(q) of (h, g) in three parts, at the place of low_g
  u32x2 b_s[NS], b_lo[NS];             // one-hot: the place of s_g, and of low_g with -16 at s_g
  uint32_t sixteens;
  float sc, slack;
  float m, msc, z;                     // of head h: the maximum, m sc, this lane's share of the sum
  float lo[NS];                        // of column (h, g): this lane's share of sum p (low - 16 s)
  f32x4 acc[8];                        // nibble n: [row 4 (l/16) + r][word l16]

  // The query rows of pair (b, hkv) on their way.
  __device__ __forceinline__ void load_q(const AttnDecArgs& a, int b, int hkv) {
    l16 = lane_id() & 15;
    g4 = lane_id() >> 4;
    h = l16 / GC;
    gl = l16 % GC;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      qr[s] = ldg16(a.q + ((int64_t)b * a.n_q + hkv * a.qpk + min(h, a.qpk - 1)) * 128 + 32 * (s * GC + gl) + 8 * g4);
  }

  // The operands that stay, for the heads `act`; nothing attended to yet.
  __device__ __forceinline__ void start(const AttnDecArgs& a, uint32_t act) {
    auto pk = [](float x, float y) { return __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xffff0000u); };
    // (scale place of group 32 g's quantisation group) = s, (low place) = low
    auto place = [&](int g, float s, float low) {
      const int slot = g / (4 / NG);
      if constexpr (NG == 4) {
        const float x = g4 & 1 ? low : s;
        return u32x2{pk(slot == 0 ? x : 0.0f, slot == 1 ? x : 0.0f), pk(slot == 2 ? x : 0.0f, slot == 3 ? x : 0.0f)};
      } else if constexpr (NG == 2) {
        return u32x2{pk(slot == 0 ? s : 0.0f, slot == 1 ? s : 0.0f),
                     pk(slot == 0 ? low : 0.0f, slot == 1 ? low : 0.0f)};
      } else {
        return u32x2{pk(s, low), 0u};
      }
    };
    const bool on = h < a.qpk && ((act >> h) & 1u);
    float mx = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        qr[s][e] = on ? qr[s][e] : 0u;
        mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(qr[s][e] << 16)), fabsf(__uint_as_float(qr[s][e] & 0xffff0000u))));
      }
    }
    if (GC >= 2) mx = fmaxf(mx, quad_xor<1>(mx));
    if (GC >= 4) mx = fmaxf(mx, quad_xor<2>(mx));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    // max |q| 2^e in [128, 256); tiny heads: as far up as the scale byte goes
    const int e2 = min(134 - (int)(__float_as_uint(mx) >> 23), 122);
    q_sc = 127 - e2;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int g = s * GC + gl;
      float x[8], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(qr[s][e] << 16);
        x[2 * e + 1] = __uint_as_float(qr[s][e] & 0xffff0000u);
        sum += x[2 * e] + x[2 * e + 1];
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y0 = __builtin_amdgcn_ldexpf(x[2 * i], e2), y1 = __builtin_amdgcn_ldexpf(x[2 * i + 1], e2);
        const int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y0, y1, 0, false);
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(32.0f * (y0 - __builtin_amdgcn_cvt_f32_fp8(hi, 0)),
                                                       32.0f * (y1 - __builtin_amdgcn_cvt_f32_fp8(hi, 1)), 0, false);
        // nibble g of word 4 (l/16) + i: byte g / 2 of the even or the odd nibbles; nibble g + 4 two bytes on
        const int sh = g & 2 ? 8 : 0;
        const int hb = ((hi & 0xff) | (hi & 0xff00) << 8) << sh, lb = ((lo & 0xff) | (lo & 0xff00) << 8) << sh;
        q_hi[s][i] = g & 1 ? 0 : hb;
        q_hi[s][4 + i] = g & 1 ? hb : 0;
        q_lo[s][i] = g & 1 ? 0 : lb;
        q_lo[s][4 + i] = g & 1 ? lb : 0;
      }
      // sum = p0 + p1 + p2, eight bits each
      const float p0 = __uint_as_float(__float_as_uint(sum) & 0xffff0000u), r1 = sum - p0;
      const float p1 = __uint_as_float(__float_as_uint(r1) & 0xffff0000u), p2 = r1 - p1;
      if constexpr (NG == 4) {
        b_low[s][0] = place(g, 0.0f, g4 == 1 ? p0 : p1);
        b_low[s][1] = place(g, 0.0f, g4 == 1 ? p2 : 0.0f);
      } else {
        b_low[s][0] = place(g, 0.0f, g4 == 0 ? p0 : g4 == 1 ? p1 : g4 == 2 ? p2 : 0.0f);
      }
      const float first = g4 < (NG == 4 ? 2 : 1) ? 1.0f : 0.0f;  // (each place counts once)
      b_s[s] = place(g, first, 0.0f);
      b_lo[s] = place(g, -16.0f * first, first);
    }
    sixteens = 0x41804180u;
    asm("" : "+v"(sixteens));
    sc = a.scale_log2;
    slack = 8.0f / sc;
    m = msc = -INFINITY;
    z = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s) lo[s] = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Keys j .. j + 31, those below j1.
  __device__ __forceinline__ void tile(int j, int j1, const Tile<NG>& T) {
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const bool odd = gl & 1, upper = gl & 2;
    i32x8 A[2];
    f32x4 x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        A[t][i] = (int)(T.kc[t][i] & 0x0f0f0f0fu);
        A[t][4 + i] = (int)((T.kc[t][i] >> 4) & 0x0f0f0f0fu);
      }
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        f32x4 D = mfma_codes(A[t], q_hi[s], zero, q_sc);
        D = mfma_codes(A[t], q_lo[s], D, q_sc - 5);
        const f32x4 ks = mfma16k16(T.km[t], b_s[s], zero);
        f32x4 y = mfma16k16(T.km[t], b_low[s][0], zero);
        if (NG == 4) y = mfma16k16(T.km[t], b_low[s][1], y);
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = fmaf(D[r], ks[r], y[r]);
        x[t] = s == 0 ? y : x[t] + y;
      }
    }
    // S[t][v]: row r = v GC + gl of half t, key 16t + 4 (l/16) + r
    float S[2][V], top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (GC == 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = x[t][r];
      } else {
        const float y0 = (odd ? x[t][1] : x[t][0]) + quad_xor<1>(odd ? x[t][0] : x[t][1]);
        const float y1 = (odd ? x[t][3] : x[t][2]) + quad_xor<1>(odd ? x[t][2] : x[t][3]);
        if constexpr (GC == 2) {
          S[t][0] = y0;
          S[t][1] = y1;
        } else {
          S[t][0] = (upper ? y1 : y0) + quad_xor<2>(upper ? y0 : y1);
        }
      }
    }
    if (j + kTile > j1) {  // the last tile
      asm volatile("");    // (a branch, not instructions in every tile)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (j + 16 * t + 4 * g4 + v * GC + gl >= j1) S[t][v] = -INFINITY;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < V; ++v) top = fmaxf(top, S[t][v]);
    if (__any(top > m + slack)) {
      if (GC >= 2) top = fmaxf(top, quad_xor<1>(top));
      if (GC >= 4) top = fmaxf(top, quad_xor<2>(top));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top), ms = mn * sc;
      const float al = mn == m ? 1.0f : __builtin_amdgcn_exp2f(msc - ms);
      m = mn;
      msc = ms;
      z *= al;
#pragma unroll
      for (int s = 0; s < NS; ++s) lo[s] *= al;
#pragma unroll
      for (int r = 0; r < 4; r += GC) {  // (a head's rows)
        const float ar = __shfl(al, 4 * g4 + r);
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[n][r + (n & 3) % GC] *= ar;
      }
    }
    u32x4 P1[NS], P2[NS];              // p s, first and second part
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float p[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        p[v] = __builtin_amdgcn_exp2f(fmaf(S[t][v], sc, -msc));
        z += p[v];
      }
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const f32x4 vs = mfma16k16(T.vm[t], b_s[s], zero), vl = mfma16k16(T.vm[t], b_lo[s], zero);
        float ps[4], rest[4];
        head_rows<GC>(p, [&](int r, float pr) {
          ps[r] = pr * vs[r];
          lo[s] = fmaf(pr, vl[r], lo[s]);
        });
#pragma unroll
        for (int r = 0; r < 4; ++r) rest[r] = ps[r] - __uint_as_float(__float_as_uint(ps[r]) & 0xffff0000u);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          P1[s][2 * t + i] =
              __builtin_amdgcn_perm(__float_as_uint(ps[2 * i + 1]), __float_as_uint(ps[2 * i]), 0x07060302u);
          P2[s][2 * t + i] = pack_bf16x2_hw(rest[2 * i], rest[2 * i + 1]);
        }
      }
    }
    // pairs of keys, nibbles 0..3 and 4..7 of the words
    uint32_t wl[4], wh[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        wl[2 * t + i] = __builtin_amdgcn_perm(T.vc[t][2 * i + 1], T.vc[t][2 * i], 0x05040100u);
        wh[2 * t + i] = __builtin_amdgcn_perm(T.vc[t][2 * i + 1], T.vc[t][2 * i], 0x07060302u);
      }
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      u32x4 B;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = n < 4 ? wl[i] : wh[i];
        B[i] = (n & 3) == 0   ? codes<0>(w, sixteens)
               : (n & 3) == 1 ? codes<1>(w, sixteens)
               : (n & 3) == 2 ? codes<2>(w, sixteens)
                              : codes<3>(w, sixteens);
      }
      acc[n] = mfma16(P1[(n & 3) / GC], B, acc[n]);
      acc[n] = mfma16(P2[(n & 3) / GC], B, acc[n]);
    }
  }

  // emit(head, maximum, sum) and store(head, dim, o[dim], o[dim + 1]) receive the
  // unnormalised result.
  template <class Emit, class Store>
  __device__ __forceinline__ void finish(const AttnDecArgs& a, Emit emit, Store store) {
    if (GC >= 2) z += quad_xor<1>(z);
    if (GC >= 4) z += quad_xor<2>(z);
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    if (g4 == 0 && gl == 0 && h < a.qpk) emit(h, msc, z);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float ls = lo[s];
      ls += __shfl_xor(ls, 16);
      ls += __shfl_xor(ls, 32);
#pragma unroll
      for (int r = 0; r < 4; ++r) {      // row (h, g) of set s
        const float l = __shfl(ls, 4 * g4 + r);
        const int g = s * GC + r % GC;
        store((4 * g4 + r) / GC, 32 * g + 2 * l16, acc[g][r] + l, acc[4 + g][r] + l);
      }
    }
  }
};

// Tiles at keys j, j + step, .. below j1 (at least one) for the heads act() of pair
// (b, hkv), through registers, two in flight.
template <int NG, int H, class Act, class Emit, class Store>
__device__ __forceinline__ void attend(const AttnDecArgs& a, int b, int hkv, Act act_of, int j, int step, int j1,
                                       Emit emit, Store store) {
  constexpr int R = 64 + 4 * NG;       // bytes of a cache row
  const int lane = lane_id(), l16 = lane & 15, g4 = lane >> 4;
  Attend<NG, H> at;
  at.load_q(a, b, hkv);
  // a view per tile of the rows up to j1; rows past them read zeros
  const uint32_t ld = a.head_major ? R : (uint32_t)a.n_kv * R;
  const int64_t base = a.head_major ? ((int64_t)b * a.n_kv + hkv) * a.L * R
                                    : (int64_t)b * a.L * ld + (int64_t)hkv * R;
  const char* kb = reinterpret_cast<const char*>(a.k) + base;
  const char* vb = reinterpret_cast<const char*>(a.v) + base;
  const uint32_t k_off = l16 * ld + 16 * g4, v_off = 4 * g4 * ld + 4 * l16;
  const uint32_t m_off = l16 * ld + 64 + (NG == 4 ? 8 * (g4 & 1) : 0);
  auto load = [&](int j, Tile<NG>& T) {
    const int n = min(max(j1 - j, 0), kTile);
    const uint32_t bytes = n > 0 ? (n - 1) * ld + R : 0;
    const int64_t at = (int64_t)j * ld;
    const bufview_t kv = buf_view(kb + at, bytes), vv = buf_view(vb + at, bytes);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      T.kc[t] = buf_ld16s(kv, k_off, 16 * t * ld);
      T.km[t] = load_meta<NG>(kv, m_off, 16 * t * ld);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        T.vc[t][r] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(vv, (int)v_off, (int)((16 * t + r) * ld), 0);
      T.vm[t] = load_meta<NG>(vv, m_off, 16 * t * ld);
    }
  };
  Tile<NG> t0, t1;
  load(j, t0);
  load(j + step, t1);
  at.start(a, act_of());
  for (; j + step < j1; j += 2 * step) {
    at.tile(j, j1, t0);
    load(j + 2 * step, t0);
    at.tile(j + step, j1, t1);
    load(j + 3 * step, t1);
  }
  if (j < j1) at.tile(j, j1, t0);
  at.finish(a, emit, store);
}

// Mask bytes of the pair's query heads, one a lane, and the heads they leave.
__device__ __forceinline__ uint8_t mask_byte(const AttnDecArgs& a, int b, int hkv) {
  return a.mask[(int64_t)b * a.ng + (hkv * a.qpk + min(lane_id(), a.qpk - 1)) / a.hpg];
}
__device__ __forceinline__ uint32_t heads_on(const AttnDecArgs& a, uint8_t on) {
  return (uint32_t)__ballot(on != 0) & ((1u << a.qpk) - 1);
}

// One workgroup of NW waves per pair.
template <int NG, int H, int NW>
__global__ __launch_bounds__(NW * 64, 2) void wide_attn_decode_kvq(AttnDecArgs a) {
  __shared__ float s_o[NW][H][128 + 4];
  __shared__ float s_m[NW][16], s_z[NW][16];
  const int w = wave_id(), p = xcd_remap(blockIdx.x, gridDim.x), b = p / a.n_kv, hkv = p - b * a.n_kv;
  const int len = seq_len(a, b);
  const uint32_t act = heads_on(a, mask_byte(a, b, hkv));
  uint32_t* out = reinterpret_cast<uint32_t*>(a.o + ((int64_t)b * a.n_q + hkv * a.qpk) * 128);
  if (act == 0 || len <= 0) {  // +0 for every head of the pair
    for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) out[i] = 0u;
    return;
  }
  if (w * kTile < len)
    attend<NG, H>(
        a, b, hkv, [&] { return act; }, w * kTile, NW * kTile, len,
        [&](int h, float m, float z) {
          s_m[w][h] = m;
          s_z[w][h] = z;
        },
        [&](int h, int d, float x, float y) { *reinterpret_cast<float2*>(&s_o[w][h][d]) = float2{x, y}; });
  __syncthreads();
  const int nw = min(NW, (len + kTile - 1) / kTile);  // waves that had a tile
  for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) {
    const int h = i >> 6, d = 2 * (i & 63);
    float mk[NW], mm = -INFINITY, zz = 0.0f, o0 = 0.0f, o1 = 0.0f;
    float2 ok[NW];
#pragma unroll
    for (int k = 0; k < NW; ++k) {  // (all of them: the reads go together; the first wave's for those without)
      const int kk = k < nw ? k : 0;
      mk[k] = k < nw ? s_m[kk][h] : -INFINITY;
      ok[k] = *reinterpret_cast<const float2*>(&s_o[kk][h][d]);
      mm = fmaxf(mm, mk[k]);
    }
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float f = k < nw ? __builtin_amdgcn_exp2f(mk[k] - mm) : 0.0f;
      zz = fmaf(f, s_z[k < nw ? k : 0][h], zz);
      o0 = fmaf(f, ok[k].x, o0);
      o1 = fmaf(f, ok[k].y, o1);
    }
    const float inv = 1.0f / zz;
    out[i] = (act >> h) & 1u ? pack_bf16x2_hw(o0 * inv, o1 * inv) : 0u;
  }
}

constexpr int kPart = 4 + 128;  // floats of a partial: maximum, sum, (two unused), o

// Equal runs of tiles a wave.
template <int NG, int H>
__global__ __launch_bounds__(kSplitThreads, 2) void wide_attn_decode_kvq_runs(AttnDecArgs a) {
  extern __shared__ uint64_t s_pre[];  // tiles and active pairs before each pair
  __shared__ uint64_t s_sum[kSplitThreads / kWave + 1];
  list_units<kTile, kKvqMinTiles>(a, s_pre, s_sum);
  auto pre = [&](int i) { return (int)(s_pre[i] & kUnitBits); };
  const int P = a.B * a.n_kv, q = __builtin_amdgcn_readfirstlane((int)s_sum[kSplitThreads / kWave]);
  const int units = __builtin_amdgcn_readfirstlane(pre(P)), wave = (int)blockIdx.x * 4 + wave_id();
  const int64_t u0 = (int64_t)wave * q;
  if (u0 >= units) return;
  const int u_end = (int)min(u0 + q, (int64_t)units);
  int p = pair_of_unit(s_pre, P, (int)u0);
  int rank = __builtin_amdgcn_readfirstlane((int)(s_pre[p] >> 40));
  int j = __builtin_amdgcn_readfirstlane(((int)u0 - pre(p)) * kTile);
  for (;; ++p, ++rank, j = 0) {
    while (pre(p + 1) == pre(p)) ++p;  // (an active pair follows: tiles are left)
    p = __builtin_amdgcn_readfirstlane(p);
    const int b = p / a.n_kv, hkv = p - b * a.n_kv;
    const int j1 = __builtin_amdgcn_readfirstlane((int)min((int64_t)seq_len(a, b), (int64_t)(u_end - pre(p)) * kTile));
    float* part = a.part + (int64_t)(wave + rank) * a.qpk * kPart;
    const uint8_t on = mask_byte(a, b, hkv);  // (loaded before the tiles, looked at after)
    attend<NG, H>(
        a, b, hkv, [&] { return heads_on(a, on); }, j, kTile, j1,
        [&](int h, float m, float z) {
          part[h * kPart] = m;
          part[h * kPart + 1] = z;
        },
        [&](int h, int d, float x, float y) {
          if (h < a.qpk) *reinterpret_cast<float2*>(part + h * kPart + 4 + d) = float2{x, y};
        });
    if (u_end <= pre(p + 1)) break;
  }
}

// Token-major caches.  A position's rows of all KV heads lie together, and a row
// ends inside a cache line where the next head's begins.  A CU holds 64 requests of
// a line each, so heads read one by one, 1.6 lines for 80 bytes, get little more
// than half of the rate (32 x 8192 keys, 8 KV heads: 98 us; 122 with the heads of a
// position on different XCDs, too, so that each fetches the line).  Here a
// workgroup of eight waves reads whole runs of rows for eight heads into LDS (71 us),
// or for four or two, the largest number that divides the heads.
//
// A unit of work is (sequence, eight KV heads, run of stages); a stage is 256 rows:
// 32 positions of eight heads, 64 of four, 128 of two.  Eight rows (of one, two or
// four positions) are a super-row, 8 R bytes; wave w of the first four loads super-rows 8 w .. 8 w + 7 of
// K, the others of V, in 16-byte chunks, direct to LDS, two stages ahead, leaving
// out chunks of inactive heads; then wave w attends for head w mod heads over the
// 32 positions of part w / heads.  The units of a sequence take q stages each, q the
// least of 64 candidates, from the mean to where the units are sure to fit, for
// which all of them fit the workgroups.
template <int NG>
struct RowStage {
  static constexpr int R = 64 + 4 * NG, SUPER = 8 * R;
  static constexpr int CK = SUPER / 16;      // chunks of a super-row
  static constexpr int CW = 8 * CK;          // chunks a wave loads
  static constexpr int LOADS = (CW + kWave - 1) / kWave;
  static constexpr int SIZE = 32 * SUPER;    // bytes of K, or V, of a stage
  static constexpr int D = 3;                // stages: K's, then V's
  static constexpr int BYTES = 2 * D * SIZE;
  // Chunk c of super-row sr lies at c - turn(sr) (mod CK), so that sixteen rows'
  // chunks of one place do not meet in a bank.  Rows of 72 and 68 bytes cross
  // chunks and stay as they are (two to four ways in a bank).
  __device__ static __forceinline__ int turn(int sr) { return NG == 4 ? (sr & 15) >> 1 : 0; }
  // byte `off` of row e of a stage
  __device__ static __forceinline__ uint32_t at(int e, int off) {
    if constexpr (NG == 4) {
      const int sr = e >> 3, c = (e & 7) * (R / 16) + off / 16 - turn(sr);
      return sr * SUPER + (c < 0 ? c + CK : c) * 16 + off % 16;
    } else {
      return e * R + off;
    }
  }
};

typedef void __attribute__((address_space(3)))* lds_t;

// Registers of a wave's tile from the stage `at` bytes into the ring.  Each group
// of reads is one asm block with its wait: before a plain LDS read the compiler
// waits for every direct-to-LDS load under way.
template <int NG>
__device__ __forceinline__ void fetch(uint32_t at, const uint32_t (&k_at)[2], const uint32_t (&km_at)[2],
                                      const uint32_t (&vm_at)[2], const uint32_t (&v_at)[2][4], Tile<NG>& T) {
  if constexpr (NG == 4) {
    asm volatile(
        "ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\tds_read_b64 %2, %8\n\t"
        "ds_read_b64 %3, %9\n\tds_read_b64 %4, %10\n\tds_read_b64 %5, %11\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(T.kc[0]), "=&v"(T.kc[1]), "=&v"(T.km[0]), "=&v"(T.km[1]), "=&v"(T.vm[0]), "=&v"(T.vm[1])
        : "v"(k_at[0] + at), "v"(k_at[1] + at), "v"(km_at[0] + at), "v"(km_at[1] + at), "v"(vm_at[0] + at),
          "v"(vm_at[1] + at)
        : "memory");
  } else if constexpr (NG == 2) {
    u32x2 k[2][2];
    asm volatile(
        "ds_read_b64 %0, %8\n\tds_read_b64 %1, %8 offset:8\n\tds_read_b64 %2, %9\n\t"
        "ds_read_b64 %3, %9 offset:8\n\tds_read_b64 %4, %10\n\tds_read_b64 %5, %11\n\t"
        "ds_read_b64 %6, %12\n\tds_read_b64 %7, %13\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(k[0][0]), "=&v"(k[0][1]), "=&v"(k[1][0]), "=&v"(k[1][1]), "=&v"(T.km[0]), "=&v"(T.km[1]),
          "=&v"(T.vm[0]), "=&v"(T.vm[1])
        : "v"(k_at[0] + at), "v"(k_at[1] + at), "v"(km_at[0] + at), "v"(km_at[1] + at), "v"(vm_at[0] + at),
          "v"(vm_at[1] + at)
        : "memory");
#pragma unroll
    for (int t = 0; t < 2; ++t) T.kc[t] = u32x4{k[t][0][0], k[t][0][1], k[t][1][0], k[t][1][1]};
  } else {
    uint32_t m[4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t k0, k1, k2, k3;
      asm volatile(
          "ds_read_b32 %0, %6\n\tds_read_b32 %1, %6 offset:4\n\tds_read_b32 %2, %6 offset:8\n\t"
          "ds_read_b32 %3, %6 offset:12\n\tds_read_b32 %4, %7\n\tds_read_b32 %5, %8\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(k0), "=&v"(k1), "=&v"(k2), "=&v"(k3), "=&v"(m[t]), "=&v"(m[2 + t])
          : "v"(k_at[t] + at), "v"(km_at[t] + at), "v"(vm_at[t] + at)
          : "memory");
      T.kc[t] = u32x4{k0, k1, k2, k3};
      T.km[t] = u32x2{m[t], 0u};
      T.vm[t] = u32x2{m[2 + t], 0u};
    }
  }
  uint32_t v[8];
  asm volatile(
      "ds_read_b32 %0, %8\n\tds_read_b32 %1, %9\n\tds_read_b32 %2, %10\n\t"
      "ds_read_b32 %3, %11\n\tds_read_b32 %4, %12\n\tds_read_b32 %5, %13\n\t"
      "ds_read_b32 %6, %14\n\tds_read_b32 %7, %15\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(v_at[0][0] + at), "v"(v_at[0][1] + at), "v"(v_at[0][2] + at), "v"(v_at[0][3] + at),
        "v"(v_at[1][0] + at), "v"(v_at[1][1] + at), "v"(v_at[1][2] + at), "v"(v_at[1][3] + at)
      : "memory");
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) T.vc[t][r] = v[4 * t + r];
}

struct HeadGroup {
  uint32_t act;  // active heads of the (up to eight) of a group
  int n;         // stages
};

// ceil(n / q) where it is far below 2^22
__device__ __forceinline__ int chunks_of(int n, int q, float inv) {
  int r = (int)((float)n * inv);
  r += n > r * q;
  r -= (r - 1) * q >= n;
  return r;
}

template <int NG, int H>
__global__ __launch_bounds__(512, 2) void wide_attn_decode_kvq_rows(AttnDecArgs a) {
  using St = RowStage<NG>;
  constexpr int NW = 8, T = NW * kWave, R = St::R;
  __shared__ __attribute__((aligned(256))) char s_ring[St::BYTES];
  __shared__ int s_cnt[NW][kWave];
  extern __shared__ HeadGroup s_grp[];
  const int tid = threadIdx.x, w = wave_id(), lane = lane_id();
  const int hg = kvq_group_heads(a.n_kv), per_seq = a.n_kv / hg, groups = a.B * per_seq;  // heads of a group, groups
  const int ks = 256 / hg;                                                      // positions of a stage

  // ---- the groups' active heads and stages
  for (int g = tid; g < groups; g += T) {
    const int len = max(seq_len(a, g / per_seq), 0);
    s_grp[g] = HeadGroup{0u, (len + ks - 1) / ks};
  }
  constexpr int MP = kKvqMaxGroups * 8 / T;  // pairs a thread
  uint32_t on = 0;  // bit k: pair tid + k T is active
  const int pairs = a.B * a.n_kv;
  auto pair_on = [&](int p) {
    const int b = p / a.n_kv, h0 = (p - b * a.n_kv) * a.qpk;
    const uint8_t* mrow = a.mask + (int64_t)b * a.ng;
    const int g0 = h0 / a.hpg, g1 = (h0 + a.qpk - 1) / a.hpg;
    uint32_t any = mrow[g0];
    for (int g = g0 + 1; g <= g1; ++g) any |= mrow[g];
    return any != 0;
  };
  for (int k = 0; k < MP && tid + k * T < pairs; ++k) on |= (uint32_t)pair_on(tid + k * T) << k;
  __syncthreads();
  for (int k = 0; k < MP; ++k)
    if ((on >> k) & 1u) {
      const int p = tid + k * T, b = p / a.n_kv, h = p - b * a.n_kv;
      atomicOr(&s_grp[b * per_seq + h / hg].act, 1u << (h & (hg - 1)));
    }
  __syncthreads();
  // all stages, and the groups that have any (every wave for itself)
  int all = 0, some = 0;
  for (int g = lane; g < groups; g += kWave) {
    const int n = s_grp[g].act ? s_grp[g].n : 0;
    all += n;
    some += n > 0;
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    all += __shfl_xor(all, d);
    some += __shfl_xor(some, d);
  }
  // q: sum ceil(n / q) <= all / q + some, so hi fits if the groups do (they are at
  // most half as many as the workgroups); 64 candidates from the mean up
  const int lo_q = max((all + a.wgs - 1) / a.wgs, 1);
  const int hi_q = max((all + a.wgs - some - 1) / (a.wgs - some), lo_q);
  int q = lo_q;
  if (hi_q > lo_q) {
    const int q_of = lo_q + (int)((int64_t)(hi_q - lo_q) * lane / (kWave - 1));
    const float inv = 1.0f / (float)q_of;
    int cnt = 0;
    for (int g = w; g < groups; g += NW) cnt += s_grp[g].act ? chunks_of(s_grp[g].n, q_of, inv) : 0;
    s_cnt[w][lane] = cnt;
    __syncthreads();
    cnt = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) cnt += s_cnt[i][lane];
    const uint64_t fits = __ballot(cnt <= a.wgs);
    q = __builtin_amdgcn_readlane(q_of, fits ? __builtin_ctzll(fits) : kWave - 1);
  }
  // this workgroup's group and run; the last workgroup writes the merge's table
  const float inv = 1.0f / (float)q;
  const bool lists = blockIdx.x == gridDim.x - 1 && w == 0;
  const int unit = blockIdx.x;
  int mine = -1, at_run = 0, before = 0;
  for (int g0 = 0; g0 < groups; g0 += kWave) {
    const int g = g0 + lane, r = g < groups && s_grp[g].act ? chunks_of(s_grp[g].n, q, inv) : 0;
    int x = r;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    const int first = before + x - r;
    const uint64_t here = __ballot(unit >= first && unit < first + r);
    if (here) {
      const int l = __builtin_ctzll(here);
      mine = g0 + l;
      at_run = unit - __builtin_amdgcn_readlane(first, l);
    }
    if (lists && g < groups)
      for (int h = 0; h < hg; ++h)  // segments of pair (group g, head h): slots 8 unit + wave
        *reinterpret_cast<int4*>(a.table + 4 * ((int64_t)g * hg + h)) =
            int4{8 * first + h, (s_grp[g].act >> h) & 1u ? r * (8 / hg) : 0, hg, 0};
    before += __builtin_amdgcn_readlane(x, kWave - 1);
  }
  if (mine < 0) return;
  const int grp = __builtin_amdgcn_readfirstlane(mine), c = __builtin_amdgcn_readfirstlane(at_run);
  const uint32_t act = __builtin_amdgcn_readfirstlane(s_grp[grp].act);
  const int n = __builtin_amdgcn_readfirstlane(s_grp[grp].n);
  const int r = __builtin_amdgcn_readfirstlane(chunks_of(n, q, inv));
  const int each = n / r, more = n - each * r, first = c * each + min(c, more);
  const int b = grp / per_seq, head0 = (grp - b * per_seq) * hg;
  const int hl = w & (hg - 1), part_of = w / hg, hkv = head0 + hl;
  int j = first * ks;
  const int j1 = __builtin_amdgcn_readfirstlane(min(max(seq_len(a, b), 0), (first + each + (c < more)) * ks));

  Attend<NG, H> at;
  at.load_q(a, b, hkv);
  const uint8_t on_byte = mask_byte(a, b, hkv);

  // ---- loads
  const int64_t ld = (int64_t)a.n_kv * R;
  const char* base = reinterpret_cast<const char*>(w < 4 ? a.k : a.v) + ((int64_t)b * a.L * a.n_kv + head0) * R;
  const int per_pos = hg * R / 16;  // chunks of a position
  uint32_t off[St::LOADS];
#pragma unroll
  for (int k = 0; k < St::LOADS; ++k) {
    const int e = min(kWave * k + lane, St::CW - 1), sr = 8 * (w & 3) + e / St::CK;
    int ch = e % St::CK + St::turn(sr);
    ch = ch >= St::CK ? ch - St::CK : ch;
    const uint32_t heads = 1u << (16 * ch / R & (hg - 1)) | 1u << ((16 * ch + 15) / R & (hg - 1));
    const int pos = (ch >= per_pos) + (ch >= 2 * per_pos) + (ch >= 3 * per_pos);  // of the super-row's 8 / hg
    off[k] = act & heads ? (uint32_t)((sr * (8 / hg) + pos) * (int)ld + 16 * (ch - pos * per_pos)) : kOffNone;
  }
  char* dst = s_ring + (w < 4 ? 0 : St::D * St::SIZE) + (w & 3) * St::CW * 16;
  auto load = [&](int j, int st) {
    const int m = min(max(j1 - j, 0), ks);
    const bufview_t view = buf_view(base + j * ld, m > 0 ? (uint32_t)((m - 1) * ld) + hg * R : 0u);
#pragma unroll
    for (int k = 0; k < St::LOADS; ++k)
      if (kWave * (k + 1) <= St::CW || kWave * k + lane < St::CW)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(view, (lds_t)(dst + st * St::SIZE + 1024 * k), 16, (int)off[k], 0, 0,
                                                 0);
  };
  load(j, 0);
  load(j + ks, 1);

  // ---- where this lane's pieces of a stage lie
  const int l16 = lane & 15, g4 = lane >> 4;
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_t)s_ring, v_lds = lds + St::D * St::SIZE;
  uint32_t k_at[2], km_at[2], vm_at[2], v_at[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int key = 32 * part_of + 16 * t, e = (key + l16) * hg + hl;
    k_at[t] = lds + St::at(e, 16 * g4);
    km_at[t] = lds + St::at(e, 64 + (NG == 4 ? 8 * (g4 & 1) : 0));
    vm_at[t] = v_lds + St::at(e, 64 + (NG == 4 ? 8 * (g4 & 1) : 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) v_at[t][i] = v_lds + St::at((key + 4 * g4 + i) * hg + hl, 4 * l16);
  }
  at.start(a, heads_on(a, on_byte));

  const bool active = (act >> hl) & 1u;
  const int off_key = 32 * part_of;
  static_assert(St::D == 3 && St::LOADS == 5, "stages");
  for (int st = 0; j < j1; j += ks) {
    t256::wait_vm<St::LOADS>();  // this wave's loads of the stage; with the barrier, all of them,
    t256::stage_barrier();       // and no one still reads the one before
    load(j + 2 * ks, st == 0 ? 2 : st - 1);
    if (active && j + off_key < j1) {
      Tile<NG> tile;
      fetch<NG>(st * St::SIZE, k_at, km_at, vm_at, v_at, tile);
      at.tile(j + off_key, j1, tile);
    }
    st = st == 2 ? 0 : st + 1;
  }
  t256::wait_vm<0>();
  if (!active) return;
  float* part = a.part + ((int64_t)unit * NW + w) * a.qpk * kPart;
  at.finish(
      a,
      [&](int h, float m, float z) {
        part[h * kPart] = m;
        part[h * kPart + 1] = z;
      },
      [&](int h, int d, float x, float y) {
        if (h < a.qpk) *reinterpret_cast<float2*>(part + h * kPart + 4 + d) = float2{x, y};
      });
}

// Joins a pair's partials: SL lanes of segments a head, each with four of the
// dimensions per lane of 32.  SL = 2: a wave a head, four heads a workgroup.
template <int SL>
__global__ __launch_bounds__(SL == 2 ? 256 : SL * 32) void wide_attn_decode_kvq_merge(AttnDecArgs a) {
  constexpr int HW = SL == 2 ? 4 : 1;
  __shared__ float s_o[SL == 2 ? 1 : SL][128 + 4], s_m[SL], s_z[SL];
  const int gh = blockIdx.x * HW + (SL == 2 ? wave_id() : 0);
  if (gh >= a.B * a.n_q) return;
  const int t = SL == 2 ? lane_id() : (int)threadIdx.x, dq = t & 31, sl = t >> 5;
  const int b = gh / a.n_q, h = gh - b * a.n_q, p = b * a.n_kv + h / a.qpk;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.o + (int64_t)gh * 128) + 2 * dq;
  // (runs: two words a pair, a segment after the other; rows: three of four, the
  // segments that far apart)
  const int32_t* tab = a.table + (a.wgs ? 4 : 2) * (int64_t)p;
  const int nseg = tab[1];
  const uint8_t on = a.mask[(int64_t)b * a.ng + h / a.hpg];
  if (!on || nseg == 0) {
    if (sl == 0) *reinterpret_cast<uint64_t*>(out) = 0;
    return;
  }
  const int64_t row = (int64_t)a.qpk * kPart, ld = a.wgs ? tab[2] * row : row;
  const float* part = a.part + tab[0] * row + (h % a.qpk) * kPart;
  float m = -INFINITY, z = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int U = SL == 32 ? 8 : 4;  // segments whose loads go together
  for (int c = sl; c < nseg; c += U * SL) {
    float cm[U], cz[U], mn = m;
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (past the end: the first one's, weight 0)
      const bool in = c + SL * u < nseg;
      const float* q = part + (in ? c + SL * u : c) * ld;
      cm[u] = in ? q[0] : -INFINITY;
      cz[u] = q[1];
      v[u] = *reinterpret_cast<const f32x4*>(q + 4 + 4 * dq);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, cm[u]);
    // (segments without a key, and lanes without a segment yet: -inf)
    const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    z *= f0;
    o *= f0;
    m = mn;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c + SL * u >= nseg) break;  // (a weight of 0 times a NaN)
      const float f = cm[u] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(cm[u] - mn);
      z = fmaf(f, cz[u], z);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[u][e], o[e]);
    }
  }
  if constexpr (SL == 2) {
    const float m2 = __shfl_xor(m, 32), mn = fmaxf(m, m2);
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    z *= f;
    o *= f;
    z += __shfl_xor(z, 32);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
    if (sl != 0) return;
  } else {
    if (dq == 0) {
      s_m[sl] = m;
      s_z[sl] = z;
    }
    *reinterpret_cast<f32x4*>(&s_o[sl][4 * dq]) = o;
    __syncthreads();
    if (t >= 64) return;
    // one wave: the lanes' weights, then four dimensions a lane over half of the lanes of segments each
    const int k = t % SL;  // (a lane without a segment: maximum -inf, sums 0)
    const float mk = s_m[k];
    float mn = mk;
#pragma unroll
    for (int d = SL / 2; d >= 1; d >>= 1) mn = fmaxf(mn, __shfl_xor(mn, d));
    const float f = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - mn);
    z = f * s_z[k];
#pragma unroll
    for (int d = SL / 2; d >= 1; d >>= 1) z += __shfl_xor(z, d);
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < SL / 2; ++i) {
      const int l = 2 * i + sl;
      const float fl = __shfl(f, l);
      const f32x4 v = *reinterpret_cast<const f32x4*>(&s_o[l][4 * dq]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(fl, v[e], o[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
    if (sl != 0) return;
  }
  const float inv = 1.0f / z;
  *reinterpret_cast<uint64_t*>(out) =
      (uint64_t)pack_bf16x2_hw(o[2] * inv, o[3] * inv) << 32 | pack_bf16x2_hw(o[0] * inv, o[1] * inv);
}

}  // namespace

constexpr int kLaunchPairs = 1 << 22;  // a workgroup each: a launch has fewer than 2^32 threads
constexpr int kShort = 64;   // tiles
constexpr int kStages = 4;   // of a workgroup
constexpr int kMany = 512;   // pairs

// How a call's work is cut (32 query heads, quantisation groups of 32; us):
//  - contexts of up to 64 tiles: a workgroup per pair.  One sequence of 1500 keys,
//    8 KV heads: 10 against 11 as runs, of 3000: 16 against 12; 64 of 1024: 16
//    against 22; token-major 32 of 2048: 22, as rows 27;
//  - token-major, an even number of KV heads (whole 16-byte pieces), more than four
//    stages of rows a workgroup: rows.  16 sequences of 4096, 8 KV heads (eight
//    stages): 25 against 35 as runs, 48 a workgroup per pair for 32 of them (43); 8
//    of 4096 (four): 20 and 18; 32 of 8192, 12 KV heads: 112, 185, 147; 10: 115, 153,
//    138.  With more than 512 groups each workgroup spends too long on the list: 900
//    sequences of 2100 682, a workgroup per pair 616; 600 of them 393 and 411;
//  - other token-major caches of more than 512 pairs: a workgroup per pair, whose
//    neighbours read the same lines at about the same time.  Which is better depends
//    on the lengths and the mask, not known here; the border is where what one side
//    gains with full sequences the other gains with ragged, half-masked ones.  3 KV
//    heads, a workgroup per pair and runs, full; ragged; ragged and half masked:
//      255 pairs, 16384 keys: 148 and 223; 126 and 121; 135 and 65
//      510 pairs, 4096 keys: 84 and 117; 63 and 68; 54 and 40
//      510 pairs, 16384 keys: 309 and 430; 227 and 236; 191 and 123
//      639 pairs, 16384 keys: 422 and 646; 272 and 293; 235 and 154
//      999 pairs, 16384 keys: 589 and 859; 378 and 464; 280 and 243;
//  - else runs.
KvqPlan attn_decode_kvq_plan(int64_t B, int n_kv, int L, int qpk, bool head_major, bool whole) {
  KvqPlan p{};
  const int hg = kvq_group_heads(n_kv);
  const int64_t pairs = B * n_kv, tiles = (L + kTile - 1) / kTile, groups = pairs / hg;
  if (tiles <= kShort || pairs * tiles > 0x7fffffff) return p;
  if (!head_major && whole && hg > 1 && tiles * pairs / 8 > kStages * kKvqWgs) {
    if (groups > kKvqMaxGroups) return p;
    // at least two workgroups a group, whole rounds of them
    p.wgs = (int)std::max<int64_t>(kKvqWgs, (2 * groups + kKvqWgs - 1) / kKvqWgs * kKvqWgs);
    p.table_ints = 4 * pairs;
    p.part_floats = (size_t)p.wgs * 8 * qpk * kPart;
  } else if (pairs <= (head_major ? kKvqMaxPairs : kMany)) {
    p.waves = kAttnDecWaves;
    p.table_ints = 2 * pairs;
    p.part_floats = (size_t)(p.waves + pairs) * qpk * kPart;
  }
  return p;
}

hipError_t launch_attention_decode_kvq(AttnDecArgs a, int quant_groups, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  const int slice = kLaunchPairs / a.n_kv;  // sequences (n_kv is at most 2^16)
  if (!a.table && a.B > slice) {
    const int64_t seq = (int64_t)a.L * a.n_kv * (64 + 4 * quant_groups) / (int64_t)sizeof *a.k;
    for (int64_t b = 0; b < a.B; b += slice) {
      AttnDecArgs part = a;
      part.B = (int)std::min<int64_t>(slice, a.B - b);
      part.q += b * a.n_q * 128;
      part.o += b * a.n_q * 128;
      part.k += b * seq;
      part.v += b * seq;
      part.mask += b * a.ng;
      if (a.kv_len) part.kv_len += b;
      const hipError_t e = launch_attention_decode_kvq(part, quant_groups, s);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  const int pairs = a.B * a.n_kv, lds = (pairs + 1) * (int)sizeof(uint64_t), groups = pairs / kvq_group_heads(a.n_kv);
#define WIDE_DEC4(NG, H)                                                                                     \
  do {                                                                                                       \
    constexpr int NW = 8;                                                                                    \
    if (a.wgs)                                                                                               \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq/rows", (wide_attn_decode_kvq_rows<NG, H>), dim3(a.wgs), dim3(512), \
                        groups * (int)sizeof(HeadGroup), s, a);                                              \
    else if (a.table)                                                                                        \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq/runs", (wide_attn_decode_kvq_runs<NG, H>), dim3(a.waves / 4), \
                        dim3(kSplitThreads), lds, s, a);                                                     \
    else                                                                                                     \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", (wide_attn_decode_kvq<NG, H, NW>), dim3(pairs), dim3(NW * 64), \
                        0, s, a);                                                                            \
  } while (0)
#define WIDE_DEC4_NG(H)                         \
  do {                                          \
    if (quant_groups == 4) WIDE_DEC4(4, H);    \
    else if (quant_groups == 2) WIDE_DEC4(2, H); \
    else WIDE_DEC4(1, H);                      \
  } while (0)
  if (a.qpk <= 4) WIDE_DEC4_NG(4);
  else if (a.qpk <= 8) WIDE_DEC4_NG(8);
  else WIDE_DEC4_NG(16);
#undef WIDE_DEC4_NG
#undef WIDE_DEC4
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.table) return e;
  const int heads = a.B * a.n_q, per = (a.wgs ? 8 * a.wgs : a.waves) / pairs;  // segments a pair, nothing masked
  // (lanes of segments 2, 8, 32, whole call in us: 8192 keys, 8 KV heads, 1 sequence
  // (256 segments) 23.1, 13.2, 11.7; 2 (128) 26.2, 15.9, 14.5; 4 (64) 21.6, 16.7, 16.7;
  // 8 (32) 24.3, 22.3, 23.0; 32 (8) 68.5, 68.4, 73.7)
  if (per > 64)
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<32>, dim3(heads), dim3(1024), 0, s, a);
  else if (per > 8)
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<8>, dim3(heads), dim3(256), 0, s, a);
  else
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<2>, dim3((heads + 3) / 4), dim3(256), 0,
                      s, a);
  return hipGetLastError();
}

}  // namespace wide
