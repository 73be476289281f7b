// Decode-step attention over a paged cache held in 8 bits: out[h] = sum_t softmax_t(scale * q[h].k[g(h),t] ks_t) * v[g(h),t] vs_t.
//
// The simplest form: a block per (sequence, KV head), a wave for every fourth token, two columns per lane.
#include "fkv_quant.h"

namespace fkv {

constexpr float kDecNegBig = -1.0e30f;

__global__ __launch_bounds__(256) void k_decode_quant(DecodeQuantArgs a) {
  constexpr int kWaves = 4;
  const DecodeArgs &d = a.d;
  __shared__ float o_lds[kWaves][kMaxReal][kHeadDim], m_lds[kWaves][kMaxReal], l_lds[kWaves][kMaxReal];
  const int b = blockIdx.x / d.Hkv, kvh = blockIdx.x % d.Hkv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = d.G;
  const int n = d.off[b + 1] - d.off[b], page_size = 1 << d.page_shift;
  const uint32_t *q = reinterpret_cast<const uint32_t *>(d.q + ((size_t)b * d.Hq + (size_t)kvh * G) * kHeadDim) + lane;
  float qx[kMaxReal], qy[kMaxReal], ox[kMaxReal] = {}, oy[kMaxReal] = {}, m[kMaxReal], l[kMaxReal] = {};
#pragma unroll
  for (int h = 0; h < kMaxReal; ++h) {
    const uint32_t w = h < G ? q[h * (kHeadDim / 2)] : 0u;
    qx[h] = __uint_as_float(w << 16);
    qy[h] = __uint_as_float(w & 0xFFFF0000u);
    m[h] = kDecNegBig;
  }
  for (int t = wave; t < n; t += kWaves) {
    const int page = min(max(d.block_table[(size_t)b * d.max_pages + (t >> d.page_shift)], 0), d.n_pages - 1);
    const size_t row = ((((size_t)page * d.Hkv + kvh) << d.page_shift)) + (t & (page_size - 1));
    const float ks = a.k_scale[row >> a.block_shift], vs = a.v_scale[row >> a.block_shift];
    const floatx2 k = __builtin_amdgcn_cvt_pk_f32_fp8(reinterpret_cast<const uint16_t *>(a.k + row * kHeadDim)[lane], false);
    const floatx2 v = __builtin_amdgcn_cvt_pk_f32_fp8(reinterpret_cast<const uint16_t *>(a.v + row * kHeadDim)[lane], false);
#pragma unroll
    for (int h = 0; h < kMaxReal; ++h) {
      if (h < G) {
        const float z = wave_fsum(qx[h] * k[0] + qy[h] * k[1]) * ks * d.scale_log2e;
        const float now = fmaxf(m[h], z), alpha = __builtin_amdgcn_exp2f(m[h] - now), p = __builtin_amdgcn_exp2f(z - now);
        m[h] = now;
        l[h] = l[h] * alpha + p;
        ox[h] = ox[h] * alpha + p * vs * v[0];
        oy[h] = oy[h] * alpha + p * vs * v[1];
      }
    }
  }
#pragma unroll
  for (int h = 0; h < kMaxReal; ++h) {
    o_lds[wave][h][2 * lane] = ox[h];
    o_lds[wave][h][2 * lane + 1] = oy[h];
    if (lane == 0) m_lds[wave][h] = m[h], l_lds[wave][h] = l[h];
  }
  __syncthreads();
  float *out = d.out + ((size_t)b * d.Hq + (size_t)kvh * G) * kHeadDim;
  for (int e = threadIdx.x; e < G * kHeadDim; e += blockDim.x) {
    const int h = e / kHeadDim, c = e % kHeadDim;
    float M = m_lds[0][h], L = 0.f, x = 0.f;
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, m_lds[w][h]);
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_lds[w][h] - M);
      L += f * l_lds[w][h];
      x += f * o_lds[w][h][c];
    }
    out[e] = n == 0 ? 0.f : L > 0.f ? x / L : __uint_as_float(0x7FC00000u);
  }
}

hipError_t launch_decode_quant(DecodeQuantArgs &a, int, hipStream_t s) {
  hipLaunchKernelGGL(k_decode_quant, dim3(a.d.n_seq * a.d.Hkv), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace fkv
