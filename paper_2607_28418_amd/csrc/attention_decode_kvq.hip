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
// One workgroup per (sequence, KV head, chunk of keys), every query head of
// the KV head packed in the MFMA's 16 columns; its waves take tiles of 32 keys
// in turn, straight into registers, and meet in LDS at the end.  Per tile, on
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
template <int NG, bool W16, int NW>
__global__ __launch_bounds__(NW * 64, 2) void wide_attn_decode_kvq(AttnDecArgs a) {
  constexpr int R = 64 + 4 * NG;       // bytes of a cache row
  constexpr int H = W16 ? 16 : 8;
  constexpr int GQ = 4 / NG;           // 32-wide groups per quantisation group
  __shared__ float s_o[NW][H][128 + 4];
  __shared__ float s_m[NW][16], s_z[NW][16], s_lo[NW][NG][16];
  const int w = wave_id(), lane = lane_id(), l16 = lane & 15, g4 = lane >> 4;
  const int item = xcd_remap(blockIdx.x, gridDim.x);
  const int p = item / a.n_chunks, chunk = item - p * a.n_chunks;
  const int b = p / a.n_kv, hkv = p - b * a.n_kv;
  const int len = a.kv_len ? min(a.kv_len[b], a.L) : a.L;
  const int j0 = chunk * a.chunk, j1 = min(len, j0 + a.chunk);
  uint32_t act = 0;
  {
    const uint8_t* mrow = a.mask + (int64_t)b * a.ng;
    for (int i = 0; i < a.qpk; ++i)
      if (mrow[(hkv * a.qpk + i) / a.hpg]) act |= 1u << i;
  }
  if (act == 0 || j0 >= j1) {
    if (a.n_chunks == 1) {  // +0 for every head of the pair
      uint32_t* o = reinterpret_cast<uint32_t*>(a.o + ((int64_t)b * a.n_q + hkv * a.qpk) * 128);
      for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) o[i] = 0u;
    }
    return;
  }

  // ---- operands that stay
  const int hc = W16 ? l16 : l16 & 7;  // this lane's head column
  u32x4 qf[4];
  float sq[4];                         // sum of q over each 32-wide group
  {
    const bool on = hc < a.qpk && ((act >> hc) & 1u);
    const uint16_t* qp = a.q + ((int64_t)b * a.n_q + hkv * a.qpk + (on ? hc : 0)) * 128 + 8 * g4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      qf[g] = on ? ldg16(qp + 32 * g) : u32x4{0, 0, 0, 0};
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

  // ---- the wave's tiles, two in flight
  constexpr int kStep = NW * kTile;
  int j = j0 + w * kTile;
  if (j < j1) {
    Tile<NG> t0, t1;
    load(j, t0);
    load(j + kStep, t1);
    for (; j + kStep < j1; j += 2 * kStep) {
      process(j, t0);
      load(j + 2 * kStep, t0);
      process(j + kStep, t1);
      load(j + 3 * kStep, t1);
    }
    if (j < j1) process(j, t0);
  }

  // ---- the waves' results meet
  z += __shfl_xor(z, 16);
  z += __shfl_xor(z, 32);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    lo[g] += __shfl_xor(lo[g], 16);
    lo[g] += __shfl_xor(lo[g], 32);
  }
  if (g4 == 0) {
    s_m[w][l16] = msc;
    s_z[w][l16] = z;
#pragma unroll
    for (int g = 0; g < NG; ++g) s_lo[w][g][l16] = lo[g];
  }
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = acc[n][r];
      if (!W16) x = __shfl_xor(x, 32) - x;  // the two parts of p s: -hi in the rows below 8
      const int h = W16 ? 4 * g4 + r : 4 * (g4 & 1) + r;
      if (W16 || g4 < 2) s_o[w][h][32 * (n & 3) + 2 * l16 + (n >> 2)] = x;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < a.qpk * 64; i += NW * 64) {
    const int h = i >> 6, d = 2 * (i & 63), g = d / (128 / NG);
    const bool on = (act >> h) & 1u;
    float mm = -INFINITY;
#pragma unroll
    for (int k = 0; k < NW; ++k) mm = fmaxf(mm, s_m[k][h]);
    float zz = 0.0f, o0 = 0.0f, o1 = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      if (j0 + k * kTile >= j1) break;  // (waves without a tile)
      const float f = __builtin_amdgcn_exp2f(s_m[k][h] - mm), l = s_lo[k][g][h];
      zz = fmaf(f, s_z[k][h], zz);
      o0 = fmaf(f, s_o[k][h][d] + l, o0);
      o1 = fmaf(f, s_o[k][h][d + 1] + l, o1);
    }
    if (a.n_chunks == 1) {
      const float inv = 1.0f / zz;
      reinterpret_cast<uint32_t*>(a.o + ((int64_t)b * a.n_q + hkv * a.qpk + h) * 128)[d / 2] =
          on ? pack_bf16x2_hw(o0 * inv, o1 * inv) : 0u;
    } else if (on) {
      float* part = a.part + ((int64_t)item * a.qpk + h) * 130;
      if (d == 0) {
        part[0] = mm;
        part[1] = zz;
      }
      part[2 + d] = o0;
      part[3 + d] = o1;
    }
  }
}

}  // namespace

// Keys per workgroup: chunks until the chip is full, none shorter than one
// round of a workgroup's waves.
int attn_decode_kvq_chunk(int64_t B, int n_kv, int L) {
  const int64_t pairs = B * n_kv;
  int ch = (L + kTile - 1) / kTile * kTile;
  while (ch > 256 && pairs * ((L + ch - 1) / ch) < 1024) ch = (ch / 2 + 127) / 128 * 128;
  return std::max(ch, kTile);
}

hipError_t launch_attention_decode_kvq(AttnDecArgs a, int quant_groups, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  constexpr int NW = 4;
  const dim3 grid((unsigned)((int64_t)a.B * a.n_kv * a.n_chunks));
#define WIDE_DEC4(NG)                                                                                              \
  do {                                                                                                             \
    if (a.qpk > 8)                                                                                                 \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", (wide_attn_decode_kvq<NG, true, NW>), grid, dim3(NW * 64), 0, s, a); \
    else                                                                                                           \
      WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", (wide_attn_decode_kvq<NG, false, NW>), grid, dim3(NW * 64), 0, s, a); \
  } while (0)
  if (quant_groups == 4) WIDE_DEC4(4);
  else if (quant_groups == 2) WIDE_DEC4(2);
  else WIDE_DEC4(1);
#undef WIDE_DEC4
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_chunks == 1) return e;
  return launch_attention_decode_merge(a, s);
}

}  // namespace wide
