// Head-group masked attention at decode over the 4-bit KV cache.
//
// The mathematics of attention_decode.hip with K and V read as codes: a row
// stands for low_g + s_g c_d in the dimensions d of group g, so
//   score  = sum_g s_g ((16 + c) . q)_g + (low_g - 16 s_g) sum(q)_g,
//   output = sum_j p_j s_jg (16 + c_jd) + p_j (low_jg - 16 s_jg).
// A bf16 with exponent 2^4 and the code in its top four mantissa bits is 16 + c
// exactly, so one shift and one and-or turn a 32-bit word of codes into two
// MFMA operands; nothing is dequantised.
//
// A wave takes tiles of 32 keys of one (sequence, KV head) pair, straight into
// registers, every query head of the KV head packed in the MFMA's 16 columns.
// Short contexts: one workgroup per pair, its waves take tiles in turn, meet in
// LDS and store o.  Longer ones: every wave takes an equal run of the active
// pairs' tiles (decode_split.h) and leaves a (maximum, sum, unnormalised o) per
// pair it meets; a second kernel joins them.  Per tile, on
// v_mfma_f32_16x16x32_bf16 unless noted:
//   scores  D_g[key][head] = (16 + c) q, a 32-wide group of dimensions each;
//           the scales as [key][head] in the same registers come from a
//           16x16x16 MFMA of the rows' (scale, low) with a one-hot operand, the
//           low terms from one with sum(q) (in three bf16 parts: 24 bits);
//   softmax online per head, fp32.  The maximum moves only when a score passes
//           it by 8 (in the exponent), so p <= 2^8, and most tiles rescale
//           nothing;
//   P.V     p s_g [head][key], straight from the scores' registers, in two
//           bf16 parts (2^-16 relative; up to 8 heads the second part sits in
//           the columns 8..15), times 16 + c; 8 columns of words a lane.
// The low terms of P.V are fp32 sums per (head, group) beside it.
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
  const uint32_t x = N == 0 ? w << 3 : w >> (4 * N - 3);
  return (x & 0x00780078u) | sixteens;
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

template <int NG>
struct Tile {
  u32x4 kc[2];   // lane: key 16t + l%16, words 4 (l/16) .. +4
  u32x2 km[2];   // lane: (scale, low) of that key
  uint32_t vc[2][4];  // lane: key 16t + 4 (l/16) + r, word l%16
  u32x2 vm[2];   // as km
};

// W16: 9..16 query heads per KV head (both parts of p s in MFMAs of their own).
// Keys j, j + 1, .. of tiles at j, j + step, .. below j1 (at least one), for
// the heads `act` of pair (b, hkv).  emit(head, maximum, sum) and
// store(head, dim, o) receive the unnormalised result.
template <int NG, bool W16, class Emit, class Store>
__device__ __forceinline__ void attend(const AttnDecArgs& a, int b, int hkv, uint32_t act, int j, int step, int j1,
                                       Emit emit, Store store) {
  constexpr int R = 64 + 4 * NG;       // bytes of a cache row
  constexpr int GQ = 4 / NG;           // 32-wide groups per quantisation group
  const int lane = lane_id(), l16 = lane & 15, g4 = lane >> 4;
  const int hc = W16 ? l16 : l16 & 7;  // this lane's head column
  u32x4 qf[4];
  {
    const bool on = hc < a.qpk && ((act >> hc) & 1u);
    const uint16_t* qp = a.q + ((int64_t)b * a.n_q + hkv * a.qpk + (on ? hc : 0)) * 128 + 8 * g4;
#pragma unroll
    for (int g = 0; g < 4; ++g) qf[g] = on ? ldg16(qp + 32 * g) : u32x4{0, 0, 0, 0};
  }
  // ---- loads: a view per tile of the rows up to j1; rows past them read zeros
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

  // ---- operands that stay
  float sq[4];                         // sum of q over each 32-wide group
  {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s += __uint_as_float(qf[g][e] << 16) + __uint_as_float(qf[g][e] & 0xffff0000u);
      s += __shfl_xor(s, 16);
      sq[g] = s + __shfl_xor(s, 32);
    }
    if constexpr (NG == 2) {
      sq[0] += sq[1];
      sq[1] = sq[2] + sq[3];
    } else if constexpr (NG == 1) {
      sq[0] = (sq[0] + sq[1]) + (sq[2] + sq[3]);
    }
  }
  // part i of x in bf16: x = part 0 + part 1 + part 2 (8 bits each)
  auto part = [](float x, int i) {
    float h = 0.0f;
    for (int k = 0; k <= i; ++k) {
      x -= h;
      h = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    }
    return h;
  };
  u32x2 b_low[2], b_s[NG], b_lo[NG];  // B operands: sum(q) terms, one-hot scale, one-hot low - 16 scale
  {
    auto pk = [](float x, float y) { return __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xffff0000u); };
    if constexpr (NG == 4) {
      const float f = g4 & 1 ? 1.0f : -16.0f;
      const int pt = g4 >> 1;
      b_low[0] = u32x2{pk(f * part(sq[0], pt), f * part(sq[1], pt)), pk(f * part(sq[2], pt), f * part(sq[3], pt))};
      const float f2 = g4 < 2 ? f : 0.0f;
      b_low[1] = u32x2{pk(f2 * part(sq[0], 2), f2 * part(sq[1], 2)), pk(f2 * part(sq[2], 2), f2 * part(sq[3], 2))};
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t sh = g & 1 ? 16 : 0;
        const uint32_t one = g4 == 0 ? 0x3f80u << sh : 0u;
        const uint32_t lo = g4 == 0 ? 0xc180u << sh : g4 == 1 ? 0x3f80u << sh : 0u;
        b_s[g] = g < 2 ? u32x2{one, 0u} : u32x2{0u, one};
        b_lo[g] = g < 2 ? u32x2{lo, 0u} : u32x2{0u, lo};
      }
    } else {
      const int pt = min(g4, 2);
      const float f = g4 < 3 ? 1.0f : 0.0f;
      if constexpr (NG == 2) {
        const float x = f * part(sq[0], pt), y = f * part(sq[1], pt);
        b_low[0] = u32x2{pk(-16.0f * x, -16.0f * y), pk(x, y)};
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const uint32_t sh = g & 1 ? 16 : 0;
          b_s[g] = u32x2{g4 == 0 ? 0x3f80u << sh : 0u, 0u};
          b_lo[g] = u32x2{g4 == 0 ? 0xc180u << sh : 0u, g4 == 0 ? 0x3f80u << sh : 0u};
        }
      } else {
        const float x = f * part(sq[0], pt);
        b_low[0] = u32x2{pk(-16.0f * x, x), 0u};
        b_s[0] = u32x2{g4 == 0 ? 0x3f80u : 0u, 0u};
        b_lo[0] = u32x2{g4 == 0 ? 0x3f80c180u : 0u, 0u};
      }
    }
  }

  const float sc = a.scale_log2, slack = 8.0f / sc;
  float m = -INFINITY, msc = -INFINITY, z = 0.0f;  // of head column hc: the maximum, m sc, this lane's share of the sum
  float lo[NG];                                    // this lane's share of sum p (low - 16 s)
  f32x4 acc[8];                                    // [head row][word l16], nibble n
#pragma unroll
  for (int g = 0; g < NG; ++g) lo[g] = 0.0f;
#pragma unroll
  for (int n = 0; n < 8; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  uint32_t sixteens = 0x41804180u;
  asm("" : "+v"(sixteens));
  const float second = !W16 && l16 >= 8 ? 1.0f : 0.0f;

  auto process = [&](int j, const Tile<NG>& T) {
    f32x4 S[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      S[t] = mfma16k16(T.km[t], b_low[0], zero);
      if (NG == 4) S[t] = mfma16k16(T.km[t], b_low[1], S[t]);
      f32x4 D[NG];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x4 A;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          A[i] = g == 0 ? codes<0>(T.kc[t][i], sixteens) : g == 1 ? codes<1>(T.kc[t][i], sixteens) : g == 2 ? codes<2>(T.kc[t][i], sixteens)
                                                                                          : codes<3>(T.kc[t][i], sixteens);
        D[g / GQ] = mfma16(A, qf[g], g % GQ == 0 ? zero : D[g / GQ]);
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const f32x4 s = mfma16k16(T.km[t], b_s[g], zero);
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = fmaf(D[g][r], s[r], S[t][r]);
      }
    }
    if (j + kTile > j1) {  // the last tile
      asm volatile("");    // (a branch, not sixteen instructions in every tile)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (j + 16 * t + 4 * g4 + r >= j1) S[t][r] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])),
                     fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
    if (__any(mx > m + slack)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m, mx), ms = mn * sc;
      const float al = mn == m ? 1.0f : __builtin_amdgcn_exp2f(msc - ms);
      m = mn;
      msc = ms;
      z *= al;
#pragma unroll
      for (int g = 0; g < NG; ++g) lo[g] *= al;
      f32x4 ar;
#pragma unroll
      for (int r = 0; r < 4; ++r) ar[r] = __shfl(al, 4 * g4 + r);
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[n][r] *= ar[r];
    }
    float P[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        P[t][r] = __builtin_amdgcn_exp2f(fmaf(S[t][r], sc, -msc));
        z += P[t][r];
      }
    // pairs of keys, nibbles 0..3 and 4..7 of the words
    uint32_t vl[4], vh[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        vl[2 * t + h] = __builtin_amdgcn_perm(T.vc[t][2 * h + 1], T.vc[t][2 * h], 0x05040100u);
        vh[2 * t + h] = __builtin_amdgcn_perm(T.vc[t][2 * h + 1], T.vc[t][2 * h], 0x07060302u);
      }
    u32x4 A, A2;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g % GQ == 0) {
        const int G = g / GQ;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const f32x4 s = mfma16k16(T.vm[t], b_s[G], zero), l = mfma16k16(T.vm[t], b_lo[G], zero);
          float x[4], y[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            lo[G] = fmaf(P[t][r], l[r], lo[G]);
            x[r] = P[t][r] * s[r];
            const float hi = __uint_as_float(__float_as_uint(x[r]) & 0xffff0000u);
            if constexpr (W16) {
              y[r] = x[r] - hi;
              x[r] = hi;
            } else {
              x[r] = fmaf(second, x[r], -hi);  // -hi, or x - hi
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            A[2 * t + h] = pack_bf16x2_hw(x[2 * h], x[2 * h + 1]);
            if constexpr (W16) A2[2 * t + h] = pack_bf16x2_hw(y[2 * h], y[2 * h + 1]);
          }
        }
      }
      u32x4 B0, B1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        B0[i] = g == 0 ? codes<0>(vl[i], sixteens) : g == 1 ? codes<1>(vl[i], sixteens) : g == 2 ? codes<2>(vl[i], sixteens) : codes<3>(vl[i], sixteens);
        B1[i] = g == 0 ? codes<0>(vh[i], sixteens) : g == 1 ? codes<1>(vh[i], sixteens) : g == 2 ? codes<2>(vh[i], sixteens) : codes<3>(vh[i], sixteens);
      }
      acc[g] = mfma16(A, B0, acc[g]);
      acc[4 + g] = mfma16(A, B1, acc[4 + g]);
      if constexpr (W16) {
        acc[g] = mfma16(A2, B0, acc[g]);
        acc[4 + g] = mfma16(A2, B1, acc[4 + g]);
      }
    }
  };

  // ---- the tiles, two in flight
  for (; j + step < j1; j += 2 * step) {
    process(j, t0);
    load(j + 2 * step, t0);
    process(j + step, t1);
    load(j + 3 * step, t1);
  }
  if (j < j1) process(j, t0);

  z += __shfl_xor(z, 16);
  z += __shfl_xor(z, 32);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    lo[g] += __shfl_xor(lo[g], 16);
    lo[g] += __shfl_xor(lo[g], 32);
  }
  if (g4 == 0 && l16 < a.qpk) emit(l16, msc, z);
  if constexpr (W16) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int n = 0; n < 8; ++n) store(4 * g4 + r, 32 * (n & 3) + 2 * l16 + (n >> 2),
                                        acc[n][r] + __shfl(lo[(n & 3) / GQ], 4 * g4 + r));
  } else {
    // the two parts of p s (rows h and 8 + h; the first with its sign turned),
    // nibbles g and g + 4 in the two halves of the wave
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[g][r]), __float_as_uint(acc[g + 4][r]),
                                                         false, false);
        const int h = 4 * (g4 & 1) + r;
        store(h, 32 * g + 2 * l16 + (g4 >> 1),
              __uint_as_float(sw[1]) - __uint_as_float(sw[0]) + __shfl(lo[g / GQ], h));
      }
  }
}

// Mask bytes of the pair's query heads, one a lane.
__device__ __forceinline__ uint32_t active_mask(const AttnDecArgs& a, int b, int hkv) {
  const int i = min(lane_id(), a.qpk - 1);
  const uint8_t on = a.mask[(int64_t)b * a.ng + (hkv * a.qpk + i) / a.hpg];
  return (uint32_t)__ballot(on != 0) & ((1u << a.qpk) - 1);
}

// One workgroup per pair.
template <int NG, bool W16, int NW>
__global__ __launch_bounds__(NW * 64, 2) void wide_attn_decode_kvq(AttnDecArgs a) {
  constexpr int H = W16 ? 16 : 8;
  __shared__ float s_o[NW][H][128 + 4];
  __shared__ float s_m[NW][16], s_z[NW][16];
  const int w = wave_id(), p = xcd_remap(blockIdx.x, gridDim.x), b = p / a.n_kv, hkv = p - b * a.n_kv;
  const int len = seq_len(a, b);
  const uint32_t act = active_mask(a, b, hkv);
  uint32_t* out = reinterpret_cast<uint32_t*>(a.o + ((int64_t)b * a.n_q + hkv * a.qpk) * 128);
  if (act == 0 || len <= 0) {  // +0 for every head of the pair
    for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) out[i] = 0u;
    return;
  }
  if (w * kTile < len)
    attend<NG, W16>(
        a, b, hkv, act, w * kTile, NW * kTile, len,
        [&](int h, float m, float z) {
          s_m[w][h] = m;
          s_z[w][h] = z;
        },
        [&](int h, int d, float x) { s_o[w][h][d] = x; });
  __syncthreads();
  const int nw = min(NW, (len + kTile - 1) / kTile);  // waves that had a tile
  for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) {
    const int h = i >> 6, d = 2 * (i & 63);
    float mm = -INFINITY;
    for (int k = 0; k < nw; ++k) mm = fmaxf(mm, s_m[k][h]);
    float zz = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int k = 0; k < nw; ++k) {
      const float f = __builtin_amdgcn_exp2f(s_m[k][h] - mm);
      zz = fmaf(f, s_z[k][h], zz);
      o0 = fmaf(f, s_o[k][h][d], o0);
      o1 = fmaf(f, s_o[k][h][d + 1], o1);
    }
    const float inv = 1.0f / zz;
    out[i] = (act >> h) & 1u ? pack_bf16x2_hw(o0 * inv, o1 * inv) : 0u;
  }
}

constexpr int kPart = 4 + 128;  // floats of a partial: maximum, sum, (two unused), o

// Equal runs of tiles a wave.
template <int NG, bool W16>
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
    const uint32_t act = active_mask(a, b, hkv);
    float* part = a.part + (int64_t)(wave + rank) * a.qpk * kPart;
    attend<NG, W16>(
        a, b, hkv, act, j, kTile, j1,
        [&](int h, float m, float z) {
          part[h * kPart] = m;
          part[h * kPart + 1] = z;
        },
        [&](int h, int d, float x) {
          if (h < a.qpk) part[h * kPart + 4 + d] = x;
        });
    if (u_end <= pre(p + 1)) break;
  }
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
  const int nseg = a.table[2 * p + 1];
  const uint8_t on = a.mask[(int64_t)b * a.ng + h / a.hpg];
  if (!on || nseg == 0) {
    if (sl == 0) *reinterpret_cast<uint64_t*>(out) = 0;
    return;
  }
  const int64_t ld = (int64_t)a.qpk * kPart;
  const float* part = a.part + a.table[2 * p] * ld + (h % a.qpk) * kPart;
  float m = -INFINITY, z = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int c = sl; c < nseg; c += 4 * SL) {
    float cm[4], cz[4];
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // four segments' loads together (past the end: the first one's, weight 0)
      const bool in = c + SL * u < nseg;
      const float* q = part + (in ? c + SL * u : c) * ld;
      cm[u] = in ? q[0] : -INFINITY;
      cz[u] = q[1];
      v[u] = *reinterpret_cast<const f32x4*>(q + 4 + 4 * dq);
    }
    const float mn = fmaxf(fmaxf(fmaxf(m, cm[0]), fmaxf(cm[1], cm[2])), cm[3]);
    const float f0 = __builtin_amdgcn_exp2f(m - mn);
    z *= f0;
    o *= f0;
    m = mn;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c + SL * u >= nseg) break;  // (a weight of 0 times a NaN)
      const float f = __builtin_amdgcn_exp2f(cm[u] - mn);
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
    if (sl != 0) return;
    const int n = min(SL, nseg);  // lanes that had a segment
    float mn = s_m[0];
    for (int k = 1; k < n; ++k) mn = fmaxf(mn, s_m[k]);
    z = 0.0f;
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < n; ++k) {
      const float f = __builtin_amdgcn_exp2f(s_m[k] - mn);
      const f32x4 v = *reinterpret_cast<const f32x4*>(&s_o[k][4 * dq]);
      z = fmaf(f, s_z[k], z);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
    }
  }
  const float inv = 1.0f / z;
  *reinterpret_cast<uint64_t*>(out) =
      (uint64_t)pack_bf16x2_hw(o[2] * inv, o[3] * inv) << 32 | pack_bf16x2_hw(o[0] * inv, o[1] * inv);
}

}  // namespace

constexpr int kShort = 48;  // tiles of a context that one workgroup takes alone

// Waves that share the work (0: one workgroup per pair).
int attn_decode_kvq_waves(int64_t B, int n_kv, int L) {
  const int64_t pairs = B * n_kv, tiles = (L + kTile - 1) / kTile;
  return pairs > kKvqMaxPairs || tiles <= kShort || pairs * tiles > 0x7fffffff ? 0 : kAttnDecWaves;
}
size_t attn_decode_kvq_part_floats(int64_t B, int n_kv, int qpk, int waves) {
  return (size_t)(waves + B * n_kv) * qpk * kPart;
}

hipError_t launch_attention_decode_kvq(AttnDecArgs a, int quant_groups, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  constexpr int NW = 8;
  const int pairs = a.B * a.n_kv, lds = (pairs + 1) * (int)sizeof(uint64_t);
#define WIDE_DEC4(NG, W16)                                                                                       \
  do {                                                                                                           \
    if (a.table)                                                                                                 \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", (wide_attn_decode_kvq_runs<NG, W16>), dim3(a.waves / 4),         \
                        dim3(kSplitThreads), lds, s, a);                                                         \
    else                                                                                                         \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", (wide_attn_decode_kvq<NG, W16, NW>), dim3(pairs), dim3(NW * 64), \
                        0, s, a);                                                                                \
  } while (0)
#define WIDE_DEC4_NG(W16)                        \
  do {                                           \
    if (quant_groups == 4) WIDE_DEC4(4, W16);    \
    else if (quant_groups == 2) WIDE_DEC4(2, W16); \
    else WIDE_DEC4(1, W16);                      \
  } while (0)
  if (a.qpk > 8) WIDE_DEC4_NG(true);
  else WIDE_DEC4_NG(false);
#undef WIDE_DEC4_NG
#undef WIDE_DEC4
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.table) return e;
  const int heads = a.B * a.n_q, per = a.waves / pairs;  // segments a pair, nothing masked
  if (per > 32)
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<32>, dim3(heads), dim3(1024), 0, s, a);
  else if (per > 8)
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<8>, dim3(heads), dim3(256), 0, s, a);
  else
    WIDE_LAUNCH_NAMED("wide_attn_decode_kvq_merge", wide_attn_decode_kvq_merge<2>, dim3((heads + 3) / 4), dim3(256), 0,
                      s, a);
  return hipGetLastError();
}

}  // namespace wide
