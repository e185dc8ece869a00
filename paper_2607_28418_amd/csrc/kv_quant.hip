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
// Both kernels are bound by memory: sixteen lanes per row, eight consecutive
// dimensions (one 16-byte load or store in bf16) each.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace wide {
namespace {

constexpr int kQT = 256;           // threads per workgroup: 16 rows
constexpr int kQRows = kQT / 16;

// Where row r of a call lies.  Token-major: rows in (token, KV head) order,
// the order of both sides.  Head-major: (KV head, token) order, so that a
// workgroup's rows are neighbours in the cache.
struct Place {
  int64_t in;      // row of the K/V tensors, (token, head) order
  int64_t cache;   // row of the cache
  bool live;       // 0 <= position < min(kv_len, L)
};
template <bool HM>
__device__ __forceinline__ Place place(const KvqArgs& a, uint32_t r) {
  const uint32_t tokens = (uint32_t)a.n_seq * (uint32_t)a.T;
  uint32_t t, h;
  if (HM) {
    h = r / tokens;
    t = r - h * tokens;
  } else {
    t = r / (uint32_t)a.n_kv;
    h = r - t * (uint32_t)a.n_kv;
  }
  const uint32_t b = t / (uint32_t)a.T;
  const int64_t p = (int64_t)(t - b * (uint32_t)a.T) + (a.pos ? a.pos[b] : 0);
  const int len = a.kv_len ? min(a.kv_len[b], a.L) : a.L;
  Place pl;
  pl.in = (int64_t)t * a.n_kv + h;
  pl.live = p >= 0 && p < len;
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
template <int N>  // row_ror:N
__device__ __forceinline__ uint32_t row_ror(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xF, 0xF, true);
}

// (greatest - low) / 15 to the nearest bf16, ties to even, in one rounding;
// 0 below 2^-126.  The fp64 quotient is never a tie that the exact one is not:
// a 53-bit w differs from 15 t by at least ulp(w), more than 15/16 of it is
// more than half an ulp of the quotient.
__device__ __forceinline__ float group_scale(double w) {
  const double q = w / 15.0;
  uint64_t u = __double_as_longlong(q);
  u += ((1ull << 44) - 1) + ((u >> 45) & 1);
  const double s = __longlong_as_double(u & ~((1ull << 45) - 1));
  return s < 0x1p-126 ? 0.0f : (float)s;
}

template <class T, int NG, bool HM>
__global__ __launch_bounds__(kQT) void wide_kv_quantize(KvqArgs a) {
  constexpr int LPG = 16 / NG;  // lanes per group
  const int i = threadIdx.x & 15, m = i >> 2, qd = i & 3;
  const T* src = static_cast<const T*>(blockIdx.y ? a.v : a.k);
  uint8_t* cache = static_cast<uint8_t*>(blockIdx.y ? a.v_cache : a.k_cache);
  const uint32_t rows = (uint32_t)a.n_seq * (uint32_t)a.T * (uint32_t)a.n_kv;
  for (uint64_t r = (uint64_t)blockIdx.x * kQRows + threadIdx.x / 16; r < rows; r += (uint64_t)gridDim.x * kQRows) {
    const Place pl = place<HM>(a, (uint32_t)r);
    if (!pl.live) continue;  // (the same for all sixteen lanes of a row)
    float x[8];
    const T* p = src + pl.in * 128 + 8 * i;
    if constexpr (sizeof(T) == 2) {
      const u32x4 w = ldg16(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    } else {
      const u32x4 w0 = ldg16(p), w1 = ldg16(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = __uint_as_float(w0[e]);
        x[4 + e] = __uint_as_float(w1[e]);
      }
    }
    float lo = x[0], hi = x[0], odd = 0.0f;  // odd: NaN where a value's double is not finite
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
      odd = fmaf(x[e] + x[e], 0.0f, odd);
    }
    lo = fminf(lo, row_xchg<1>(lo)); hi = fmaxf(hi, row_xchg<1>(hi)); odd += row_xchg<1>(odd);
    lo = fminf(lo, row_xchg<2>(lo)); hi = fmaxf(hi, row_xchg<2>(hi)); odd += row_xchg<2>(odd);
    odd += row_xchg<4>(odd);
    odd += row_xchg<8>(odd);
    if (LPG >= 8) { lo = fminf(lo, row_xchg<4>(lo)); hi = fmaxf(hi, row_xchg<4>(hi)); }
    if (LPG >= 16) { lo = fminf(lo, row_xchg<8>(lo)); hi = fmaxf(hi, row_xchg<8>(hi)); }
    uint32_t lbits = __float_as_uint(lo);
    if (sizeof(T) == 4) {  // towards -inf: a negative number's size grows for the bits cut off
      const uint32_t cut = lbits & 0xffff0000u;
      lbits = (lbits >> 31) && cut != lbits ? cut + 0x10000u : cut;
    }
    const double low = (double)__uint_as_float(lbits);
    float s = group_scale((double)hi - low);
    if (odd != 0.0f) {  // (NaN)
      s = 0.0f;
      lbits = 0x7fc00000u;
    }
    const float inv = s > 0.0f ? 1.0f / s : 0.0f, lf = __uint_as_float(lbits);
    const double sd = (double)s, half = 0.5 * sd;
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // the nearest code up to fp32 rounding, then the exact remainder decides
      float kf = rintf((x[e] - lf) * inv);
      kf = s > 0.0f ? fminf(fmaxf(kf, 0.0f), 15.0f) : 0.0f;
      const double rem = fma(-sd, (double)kf, (double)x[e] - low);
      int c = (int)kf;
      if (s > 0.0f && (fabs(rem) > half || (fabs(rem) == half && (c & 1)))) c += rem > 0.0 ? 1 : -1;
      code[e] = (uint32_t)min(max(c, 0), 15);
    }
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = (code[2 * e] | code[2 * e + 1] << 16) << (4 * m);
      w[e] |= row_ror<4>(w[e]);
      w[e] |= row_ror<8>(w[e]);
    }
    uint8_t* row = cache + pl.cache * (64 + 4 * NG);
    const uint32_t mine = m == 0 ? w[0] : m == 1 ? w[1] : m == 2 ? w[2] : w[3];
    *reinterpret_cast<uint32_t*>(row + 16 * qd + 4 * m) = mine;
    if (i % LPG == 0) {
      uint16_t* meta = reinterpret_cast<uint16_t*>(row + 64);
      meta[i / LPG] = (uint16_t)(__float_as_uint(s) >> 16);
      meta[NG + i / LPG] = (uint16_t)(lbits >> 16);
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
  const uint32_t rows = (uint32_t)a.n_seq * (uint32_t)a.T * (uint32_t)a.n_kv;
  for (uint64_t r = (uint64_t)blockIdx.x * kQRows + threadIdx.x / 16; r < rows; r += (uint64_t)gridDim.x * kQRows) {
    const Place pl = place<HM>(a, (uint32_t)r);
    float y[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (pl.live) {
      const uint8_t* row = cache + pl.cache * (64 + 4 * NG);
      const u32x4 w = *reinterpret_cast<const u32x4_a4*>(row + 16 * qd);
      const uint16_t* meta = reinterpret_cast<const uint16_t*>(row + 64);
      const float s = bf16_to_f32(meta[i / LPG]), low = bf16_to_f32(meta[NG + i / LPG]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t c = w[e] >> (4 * m);
        y[2 * e] = fmaf(s, (float)(c & 15u), low);
        y[2 * e + 1] = fmaf(s, (float)(c >> 16 & 15u), low);
      }
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

hipError_t launch_kv_quant(const KvqArgs& a, bool f32, bool read, hipStream_t s) {
  const int64_t rows = a.n_seq * a.T * a.n_kv;
  if (rows == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((rows + kQRows - 1) / kQRows, 1 << 20), 2);
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
