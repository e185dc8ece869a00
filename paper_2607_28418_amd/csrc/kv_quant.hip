// The 4-bit KV cache on gfx950: rows quantised as they are written, and read
// back.
//
// A cache row (one sequence, position and KV head: 128 dimensions) is
//   64 bytes of codes | ng bf16 scales | ng bf16 lows      (ng = 128 / quant_group)
// and a code c of group g stands for low[g] + scale[g] * c.  Word l (16
// little-endian words) holds dimension 32 (n mod 4) + 2 l + n / 4 in nibble n:
// one shift and one mask then leave two adjacent dimensions of one 32-wide
// group in the halves of a register (the K operand of a 16x16x32 MFMA in
// natural order), and nibble n belongs to the same group in every word (the
// V operand, whose columns are the words).
//
// Quantisation of a group: low = its least value rounded down to bf16 (exact
// for bf16 rows), scale = (greatest - low) / 15 rounded to nearest bf16, code =
// (x - low) / scale rounded to nearest, all decided exactly (ties to even), so
// a value next to the border of two codes always gets the nearer one.  A scale
// below 2^-126 becomes 0, and its group reads back as low.  A row that holds a
// NaN, an infinity or a magnitude of 2^127 or more reads back as NaN (below that
// no low, scale or value read back overflows).
//
// Sixteen lanes per row, eight consecutive dimensions (one 16-byte load or store
// in bf16) each; many small workgroups hide the loads (two or four rows a lane,
// loaded together, ran 8-15% slower).  Reading back is bound by memory (8 x 32768
// positions of 8 heads in bf16, 1.36 GB: 270 us, 5.0 TB/s, the rate of a copy);
// quantising by the vector ALUs: 210 instructions a lane, 11 of the 13 us that 8192
// positions of 8 heads take in bf16 (44 MB, 3.3 TB/s).  Exact decisions are five
// fp32 operations an element where every x - low is exact (nearly always, in bf16;
// all of it in fp64 took 22 us), fp64 and what its differences lose elsewhere.  fp32
// rows take the fp64 arm: the same positions (78 MB) 18 us.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace wide {
namespace {

constexpr int kQT = 256;           // threads per workgroup
constexpr int kQRows = kQT / 16;   // rows of a row block

// n / d for n < 2^31 (d from 1 to 2^31 - 1): Granlund and Montgomery's
// multiplication by a rounded-up reciprocal.
__device__ __forceinline__ uint32_t div_by(uint32_t n, FastDiv f) { return (__umulhi(f.mul, n) + n) >> f.shift; }

// Where this lane's row of row block `blk` lies (sixteen rows).  Token-major:
// rows in (token, KV head) order, the order of both sides.  Head-major: sixteen
// tokens of one head, neighbours in the cache, the heads in turn so that
// workgroups side by side touch whole rows of the K/V tensors (one head after
// the other wrote one eighth of every 4 KB: 19 us instead of 15 for 8192 fp32
// rows of 8 heads).
struct Place {
  int64_t in;      // row of the K/V tensors, (token, head) order
  int64_t cache;   // row of the cache
  bool some;       // there is such a row
  bool live;       // and 0 <= position < min(kv_len, L)
};
template <bool HM>
__device__ __forceinline__ Place place(const KvqArgs& a, uint32_t blk) {
  const uint32_t tokens = (uint32_t)(a.n_seq * a.T), sub = threadIdx.x / 16;
  uint32_t t, h;
  Place pl;
  if (HM) {
    const uint32_t tile = div_by(blk, a.by_heads);
    h = blk - tile * (uint32_t)a.n_kv;
    t = tile * kQRows + sub;
  } else {
    const uint32_t r = min(blk * kQRows + sub, tokens * (uint32_t)a.n_kv);  // (past the last block: no row)
    t = div_by(r, a.by_heads);
    h = r - t * (uint32_t)a.n_kv;
  }
  pl.some = t < tokens;
  t = min(t, tokens - 1);
  const uint32_t b = div_by(t, a.by_T);
  const int64_t p = (int64_t)(t - b * (uint32_t)a.T) + (a.pos ? a.pos[b] : 0);
  const int len = a.kv_len ? min(a.kv_len[b], a.L) : a.L;
  pl.in = (int64_t)t * a.n_kv + h;
  pl.live = pl.some && p >= 0 && p < len;
  pl.cache = HM ? ((int64_t)b * a.n_kv + h) * a.L + p : ((int64_t)b * a.L + p) * a.n_kv + h;
  return pl;
}

// Value of lane l ^ D of each 16-lane row (D = 1, 2), or of the other half of
// the 8- or 16-lane block (D = 4, 8: mirrored; used on values that are already
// equal over that half).
template <int D>
__device__ __forceinline__ float row_xchg(float x) {
  constexpr int ctrl = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x140;
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xF, 0xF, true));
}
template <int D>
__device__ __forceinline__ uint32_t row_xchg_u(uint32_t x) {
  return __float_as_uint(row_xchg<D>(__uint_as_float(x)));
}
template <int N>  // row_ror:N
__device__ __forceinline__ uint32_t row_ror(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xF, 0xF, true);
}

// a - b = d + this, exactly (d the rounded difference; Knuth's two-sum).
__device__ __forceinline__ double diff_rest(double a, double b, double d) {
  const double v = a - d;
  return (a - (d + v)) + (v - b);
}

// (w + rest) / 15 to the nearest bf16, ties to even, in one rounding; 0 below
// 2^-126.  The fp64 quotient w / 15 is never a tie that the exact one is not:
// a 53-bit w differs from 15 t by at least ulp(w), more than 15/16 of it is
// more than half an ulp of the quotient.  rest, half an ulp of w at most, counts
// where w is such a 15 t.
__device__ __forceinline__ float group_scale(double w, double rest) {
  const double q = w / 15.0;
  uint64_t u = __double_as_longlong(q);
  u += ((1ull << 44) - 1) + (rest == 0.0 ? (u >> 45) & 1 : rest > 0.0);
  const double s = __longlong_as_double(u & ~((1ull << 45) - 1));
  return s < 0x1p-126 ? 0.0f : (float)s;
}

// What a lane finds of its eight values x: their group's scale and low (bf16 bits)
// and the codes, two a word (16 bits each).  NaN groups: scale 0, low NaN.
struct Coded {
  uint32_t scale, low, code[4];
};

// Every step in fp64 where a rounding could change a decision, and what a
// difference of values 2^45 apart loses there.
template <bool CUT>
__device__ __forceinline__ Coded code_fp64(const float (&x)[8], float lo, float hi, bool bad) {
  uint32_t lbits = __float_as_uint(lo);
  if (CUT) {  // towards -inf: a negative number's size grows for the bits cut off
    const uint32_t cut = lbits & 0xffff0000u;
    lbits = (lbits >> 31) && cut != lbits ? cut + 0x10000u : cut;
  }
  const double low = (double)__uint_as_float(lbits);
  const double w = (double)hi - low;
  const float s = bad ? 0.0f : group_scale(w, diff_rest(hi, low, w));
  const float inv = s > 0.0f ? 1.0f / s : 0.0f, lf = __uint_as_float(lbits);
  const double sd = (double)s, half = 0.5 * sd;
  uint32_t code[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // the nearest code up to fp32 rounding, then the remainder decides.  The
    // difference d, and so the remainder, may lack half an ulp of d, which counts
    // on the border only: d is at most 16 s, so both sides of the comparison are
    // multiples of that ulp.
    float kf = rintf((x[e] - lf) * inv);
    kf = s > 0.0f ? fminf(fmaxf(kf, 0.0f), 15.0f) : 0.0f;
    const double d = (double)x[e] - low, rem = fma(-sd, (double)kf, d);
    int c = (int)kf;
    if (s > 0.0f && fabs(rem) >= half) {
      const double rest = diff_rest(x[e], low, d);
      if (fabs(rem) > half || (rest == 0.0 ? (c & 1) != 0 : (rest > 0.0) == (rem > 0.0))) c += rem > 0.0 ? 1 : -1;
    }
    code[e] = (uint32_t)min(max(c, 0), 15);
  }
  Coded o;
  o.scale = __float_as_uint(s) >> 16;
  o.low = bad ? 0x7fc0u : lbits >> 16;
#pragma unroll
  for (int e = 0; e < 4; ++e) o.code[e] = code[2 * e] | code[2 * e + 1] << 16;
  return o;
}

// The same decisions in fp32 for bf16 values whose differences x - low, and
// hi - low, are exact.  With w and t = x - low exact in 24 bits and s in 8, the
// correctly rounded quotients w / 15 and t / s never fall on a border (between
// two bf16 values, between two codes) that the exact ones do not: a numerator
// that misses the border's multiple misses it by an ulp of its own, and an ulp
// over s < 2^(e+1), or over 15 < 2^4, is more than half an ulp of the quotient.
// q + r / s with r the exact remainder is that quotient (Markstein).
__device__ __forceinline__ Coded code_fp32(const float (&x)[8], float lo, float hi) {
  const float w = hi - lo, c15 = 1.0f / 15.0f, q15 = w * c15;
  uint32_t sb = __float_as_uint(fmaf(fmaf(-15.0f, q15, w), c15, q15));
  sb = (sb + 0x7fffu + ((sb >> 16) & 1u)) & 0xffff0000u;
  const float s = __uint_as_float(sb), inv = s > 0.0f ? 1.0f / s : 0.0f;
  uint32_t k[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = x[e] - lo, q = t * inv;
    k[e] = __float_as_uint(fmaf(fmaf(-s, q, t), inv, q) + 0x1.8p23f);  // the code in the low bits, ties to even
  }
  Coded o;
  o.scale = sb >> 16;
  o.low = __float_as_uint(lo) >> 16;
#pragma unroll
  for (int e = 0; e < 4; ++e) o.code[e] = __builtin_amdgcn_perm(k[2 * e + 1], k[2 * e], 0x05040100u);
  return o;
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 min2(u16x2 a, u16x2 b) { return __builtin_elementwise_min(a, b); }
__device__ __forceinline__ u16x2 max2(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }

template <class T, int NG, bool HM>
__global__ __launch_bounds__(kQT) void wide_kv_quantize(KvqArgs a) {
  constexpr int LPG = 16 / NG;  // lanes per group
  constexpr bool F32 = sizeof(T) == 4;
  const int i = threadIdx.x & 15, m = i >> 2, qd = i & 3;
  const T* src = static_cast<const T*>(blockIdx.y ? a.v : a.k);
  uint8_t* cache = static_cast<uint8_t*>(blockIdx.y ? a.v_cache : a.k_cache);
  for (uint32_t blk = blockIdx.x; blk < a.blocks; blk += gridDim.x) {
    const Place pl = place<HM>(a, blk);
    if (!pl.live) continue;  // (the same for all sixteen lanes of a row)
    const T* p = src + pl.in * 128 + 8 * i;
    u32x4 w[F32 ? 2 : 1];
    w[0] = ldg16(p);
    if constexpr (F32) w[1] = ldg16(p + 4);
    float x[8];
    bool bad, wide;  // a value at 2^127 or beyond, or not a number; differences that may not be exact
    if constexpr (F32) {
      float odd = 0.0f;  // NaN where a value's double is not finite
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = __uint_as_float(w[e / 4][e % 4]);
        odd = fmaf(x[e] + x[e], 0.0f, odd);
      }
      odd += row_xchg<1>(odd);
      odd += row_xchg<2>(odd);
      odd += row_xchg<4>(odd);
      odd += row_xchg<8>(odd);
      bad = odd != 0.0f;
      wide = true;
    } else {
      u16x2 big = {0, 0}, small = {0xffff, 0xffff};  // of the sizes; zeros wrap to the top for the least
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[0][e] << 16);
        x[2 * e + 1] = __uint_as_float(w[0][e] & 0xffff0000u);
        const u16x2 size = __builtin_bit_cast(u16x2, w[0][e] & 0x7fff7fffu);
        big = max2(big, size);
        small = min2(small, size - (u16x2){1, 1});
      }
      uint32_t top = max(big[0], big[1]), least = min(small[0], small[1]);
      top = max(top, row_xchg_u<1>(top)); least = min(least, row_xchg_u<1>(least));
      top = max(top, row_xchg_u<2>(top)); least = min(least, row_xchg_u<2>(least));
      top = max(top, row_xchg_u<4>(top)); least = min(least, row_xchg_u<4>(least));
      top = max(top, row_xchg_u<8>(top)); least = min(least, row_xchg_u<8>(least));
      bad = top >= 0x7f00u;
      // exact while no size is below 2^-15 of the row's largest, which is not
      // near the smallest numbers (2^-60: the remainders are exact, too)
      wide = bad || top < (67u << 7) || least + 1 < top - (15u << 7);
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
    }
    lo = fminf(lo, row_xchg<1>(lo)); hi = fmaxf(hi, row_xchg<1>(hi));
    lo = fminf(lo, row_xchg<2>(lo)); hi = fmaxf(hi, row_xchg<2>(hi));
    if (LPG >= 8) { lo = fminf(lo, row_xchg<4>(lo)); hi = fmaxf(hi, row_xchg<4>(hi)); }
    if (LPG >= 16) { lo = fminf(lo, row_xchg<8>(lo)); hi = fmaxf(hi, row_xchg<8>(hi)); }
    Coded c;
    if (wide) c = code_fp64<F32>(x, lo, hi, bad);
    else c = code_fp32(x, lo, hi);
    // word 4 qd + e of the row: nibbles m and m + 4 from this lane, the other
    // groups' from the lanes four, eight and twelve away
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = c.code[e] << (4 * m);
      v[e] |= row_ror<4>(v[e]);
      v[e] |= row_ror<8>(v[e]);
    }
    uint8_t* row = cache + pl.cache * (64 + 4 * NG);
    const uint32_t mine = m == 0 ? v[0] : m == 1 ? v[1] : m == 2 ? v[2] : v[3];
    *reinterpret_cast<uint32_t*>(row + 16 * qd + 4 * m) = mine;
    if (i % LPG == 0) {
      uint16_t* meta = reinterpret_cast<uint16_t*>(row + 64);
      meta[i / LPG] = (uint16_t)c.scale;
      meta[NG + i / LPG] = (uint16_t)c.low;
    }
  }
}

typedef u32x4 __attribute__((aligned(4))) u32x4_a4;

template <class T, int NG, bool HM>
__global__ __launch_bounds__(kQT) void wide_kv_dequantize(KvqArgs a) {
  constexpr int LPG = 16 / NG;
  const int i = threadIdx.x & 15, m = i >> 2, qd = i & 3;
  T* dst = static_cast<T*>(const_cast<void*>(blockIdx.y ? a.v : a.k));
  const uint8_t* cache = static_cast<const uint8_t*>(blockIdx.y ? a.v_cache : a.k_cache);
  for (uint32_t blk = blockIdx.x; blk < a.blocks; blk += gridDim.x) {
    const Place pl = place<HM>(a, blk);
    if (!pl.some) continue;
    u32x4 w = {0, 0, 0, 0};
    uint16_t sb = 0, lb = 0;
    if (pl.live) {
      const uint8_t* row = cache + pl.cache * (64 + 4 * NG);
      w = *reinterpret_cast<const u32x4_a4*>(row + 16 * qd);
      const uint16_t* meta = reinterpret_cast<const uint16_t*>(row + 64);
      sb = meta[i / LPG];
      lb = meta[NG + i / LPG];
    }
    const float s = bf16_to_f32(sb), low = bf16_to_f32(lb);
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t c = w[e] >> (4 * m);
      y[2 * e] = fmaf(s, (float)(c & 15u), low);
      y[2 * e + 1] = fmaf(s, (float)(c >> 16 & 15u), low);
    }
    T* p = dst + pl.in * 128 + 8 * i;
    if constexpr (sizeof(T) == 2) {
      stg16(p, u32x4{pack_bf16x2_hw(y[0], y[1]), pack_bf16x2_hw(y[2], y[3]), pack_bf16x2_hw(y[4], y[5]),
                     pack_bf16x2_hw(y[6], y[7])});
    } else {
      stg16(p, __builtin_bit_cast(u32x4, f32x4{y[0], y[1], y[2], y[3]}));
      stg16(p + 4, __builtin_bit_cast(u32x4, f32x4{y[4], y[5], y[6], y[7]}));
    }
  }
}

}  // namespace

static FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (uint64_t(1) << l) < d) ++l;
  return FastDiv{(uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1), l};
}

hipError_t launch_kv_quant(KvqArgs a, bool f32, bool read, hipStream_t s) {
  const int64_t tokens = a.n_seq * a.T;
  if (tokens == 0) return hipSuccess;
  a.by_heads = fast_div((uint32_t)a.n_kv);
  a.by_T = fast_div((uint32_t)a.T);
  a.blocks = (uint32_t)(a.head_major ? (tokens + kQRows - 1) / kQRows * a.n_kv
                                     : (tokens * a.n_kv + kQRows - 1) / kQRows);
  const dim3 grid(std::min(a.blocks, 1u << 22), 2);
#define WIDE_KVQ(T, NG, HM)                                                                               \
  do {                                                                                                    \
    if (read) WIDE_LAUNCH_NAMED("wide_kv_dequantize", (wide_kv_dequantize<T, NG, HM>), grid, dim3(kQT), 0, s, a); \
    else WIDE_LAUNCH_NAMED("wide_kv_quantize", (wide_kv_quantize<T, NG, HM>), grid, dim3(kQT), 0, s, a);  \
  } while (0)
#define WIDE_KVQ_NG(T, HM)                \
  do {                                    \
    if (a.ng == 4) WIDE_KVQ(T, 4, HM);    \
    else if (a.ng == 2) WIDE_KVQ(T, 2, HM); \
    else WIDE_KVQ(T, 1, HM);              \
  } while (0)
  if (f32) {
    if (a.head_major) WIDE_KVQ_NG(float, true);
    else WIDE_KVQ_NG(float, false);
  } else {
    if (a.head_major) WIDE_KVQ_NG(uint16_t, true);
    else WIDE_KVQ_NG(uint16_t, false);
  }
#undef WIDE_KVQ_NG
#undef WIDE_KVQ
  return hipGetLastError();
}

}  // namespace wide
