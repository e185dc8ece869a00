// Head-group masked attention at decode over the 4-bit KV cache.
//
// The mathematics of attention_decode.hip with K and V read as codes: a key
// row stands for lo_g + s_g c_d in the dimensions of group g, so
//   score  = sum_g s_g (c . q)_g + lo_g sum(q)_g,
//   output = sum_j p_j (lo_jg + s_jg c_jd).
//
// One wave per (sequence, query head, key chunk): lane = byte l % 4 of code
// word l / 4, two dimensions.  A (max, sum, unnormalised o) per chunk is left
// for the merge kernel that the bf16 cache's decode attention uses.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace wide {
namespace {

template <int NG>
__global__ __launch_bounds__(256) void wide_attn_decode_kvq(AttnDecArgs a) {
  constexpr int R = 64 + 4 * NG, QG = 128 / NG;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave_id();
  if (item >= (int64_t)a.B * a.n_q * a.n_chunks) return;
  const int c = (int)(item % a.n_chunks), h = (int)(item / a.n_chunks % a.n_q), b = (int)(item / a.n_chunks / a.n_q);
  const int hkv = h / a.qpk;
  if (!a.mask[(int64_t)b * a.ng + h / a.hpg]) return;
  const int len = a.kv_len ? min(a.kv_len[b], a.L) : a.L;
  const int j0 = c * a.chunk, j1 = min(len, j0 + a.chunk);
  if (j0 >= j1) return;
  const int lane = lane_id(), word = lane >> 2, byte = lane & 3;
  const int d0 = 32 * (2 * byte % 4) + 2 * word + byte / 2, d1 = d0 + 32;
  const uint16_t* q = a.q + ((int64_t)b * a.n_q + h) * 128;
  const float q0 = bf16_to_f32(q[d0]) * a.scale_log2, q1 = bf16_to_f32(q[d1]) * a.scale_log2;
  const int64_t ld = a.head_major ? R : (int64_t)a.n_kv * R;
  const int64_t base = a.head_major ? ((int64_t)b * a.n_kv + hkv) * a.L * R : (int64_t)b * a.L * ld + (int64_t)hkv * R;
  const uint8_t* kp = reinterpret_cast<const uint8_t*>(a.k) + base;
  const uint8_t* vp = reinterpret_cast<const uint8_t*>(a.v) + base;
  auto value = [&](const uint8_t* row, float& x0, float& x1) {
    const uint32_t cc = row[lane];
    const uint16_t* meta = reinterpret_cast<const uint16_t*>(row + 64);
    x0 = fmaf(bf16_to_f32(meta[d0 / QG]), (float)(cc & 15u), bf16_to_f32(meta[NG + d0 / QG]));
    x1 = fmaf(bf16_to_f32(meta[d1 / QG]), (float)(cc >> 4), bf16_to_f32(meta[NG + d1 / QG]));
  };
  float mx = -INFINITY, z = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int j = j0; j < j1; ++j) {
    float k0, k1, v0, v1;
    value(kp + j * ld, k0, k1);
    value(vp + j * ld, v0, v1);
    float sc = fmaf(q0, k0, q1 * k1);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sc += __shfl_xor(sc, o);
    const float mn = fmaxf(mx, sc), al = __builtin_amdgcn_exp2f(mx - mn), p = __builtin_amdgcn_exp2f(sc - mn);
    z = fmaf(z, al, p);
    o0 = fmaf(o0, al, p * v0);
    o1 = fmaf(o1, al, p * v1);
    mx = mn;
  }
  float* part = a.part + (((int64_t)(b * a.n_kv + hkv) * a.n_chunks + c) * a.qpk + h % a.qpk) * 130;
  if (lane == 0) {
    part[0] = mx;
    part[1] = z;
  }
  part[2 + d0] = o0;
  part[2 + d1] = o1;
}

}  // namespace

int attn_decode_kvq_chunk(int64_t B, int n_kv, int L) {
  int ch = 2048;
  while (ch > 64 && B * n_kv * ((L + ch - 1) / ch) < 2048) ch /= 2;
  return ch;
}

hipError_t launch_attention_decode_kvq(AttnDecArgs a, int quant_groups, hipStream_t s) {
  if (a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)(((int64_t)a.B * a.n_q * a.n_chunks + 3) / 4));
  if (quant_groups == 4) WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", wide_attn_decode_kvq<4>, grid, dim3(256), 0, s, a);
  else if (quant_groups == 2) WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", wide_attn_decode_kvq<2>, grid, dim3(256), 0, s, a);
  else WIDE_LAUNCH_NAMED("wide_attn_decode_kvq", wide_attn_decode_kvq<1>, grid, dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_attention_decode_merge(a, s);
}

}  // namespace wide
