// What the decode kernels share: the shares of their work, a row's pieces and their fold.
#pragma once

#include "fkv_dpp.h"
#include "fkv_internal.h"

namespace fkv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;

constexpr int kDecTile = 32;                  // tokens a wave works on at a time
constexpr float kDecNegBig = -1.0e30f;

__device__ __forceinline__ float dec_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The sum a row is divided by.  Zero: no token has a finite logit and the softmax no value; NaN then, and not what the
// kept-up pieces of the probabilities (see k_decode) divided by zero would give.
__device__ __forceinline__ float row_sum(float l) { return l > 0.f ? l : __uint_as_float(0x7FC00000u); }

__device__ __forceinline__ void agent_store2(float *p, float x, float y) {
  const float2 v = make_float2(x, y);
  unsigned long long bits;
  __builtin_memcpy(&bits, &v, sizeof bits);
  __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 agent_load2(const float *p) {
  const unsigned long long bits =
      __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  float2 v;
  __builtin_memcpy(&v, &bits, sizeof v);
  return v;
}

// The work of a launch is a line of 32-token tiles, row after row (a row = one KV head of one sequence); block i
// of N takes tiles [i T / N, (i + 1) T / N).  A row that lies inside one block is finished there; the pieces of a row
// that is cut go to partial slots, at most two per block (2 i: a piece that does not begin its row, 2 i + 1: one that does).
// T < 2^30; the products of these bounds are not, so they are formed from quotient and remainder.
__device__ __forceinline__ uint32_t share_at(uint32_t len, uint32_t part, uint32_t parts) {  // len * part / parts
  const uint32_t per = len / parts, rem = len - per * parts;
  return part * per + part * rem / parts;
}
__device__ __forceinline__ int dec_block_of(uint64_t tile, uint64_t tiles, uint64_t n_blocks) {
  return (int)(((tile + 1) * n_blocks - 1) / tiles);
}

// Folds the n_split pieces of a row, whose first lies in block blk0, into out [G][d]: one wave per head, two columns per lane.
template <bool kAligned, int kWaves>
__device__ __forceinline__ void fold_row(const DecodeArgs &a, int blk0, int n_split, float *out) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = a.G;
  // equal shares: piece p of the row lies in block blk0 + p; only the first one begins the row
  const float *src = a.part + 2 * (size_t)blk0 * kDecodeSlotFloats;
  auto piece = [&](int p) { return src + (size_t)(kAligned ? 2 * p * a.Hkv : p == 0 ? 1 : 2 * p) * kDecodeSlotFloats; };
  constexpr int kBatch = 16;  // partial rows in flight per lane
  for (int h = wave; h < G; h += kWaves) {
    const float2 ml = agent_load2(piece(min(lane, n_split - 1)) + kMaxReal * kHeadDim + 2 * h);
    float2 v[kBatch];
    auto request = [&](int s0) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) v[i] = agent_load2(piece(min(s0 + i, n_split - 1)) + h * kHeadDim + 2 * lane);
    };
    request(0);
    // the pieces' weights, a lane each
    const float mp = lane < n_split ? ml.x : kDecNegBig;
    const float f = dec_exp2(mp - wave_fmax(mp));
    const float L = row_sum(wave_fsum(lane < n_split ? ml.y * f : 0.f));
    const int weight = __float_as_int(lane < n_split ? f / L : 0.f);
    float x = 0.f, y = 0.f;
    for (int s0 = 0; s0 < n_split; s0 += kBatch) {
      if (s0 > 0) request(s0);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {  // past the last piece nothing is added: 0 times an infinite sum would be NaN
        const float w = __int_as_float(__builtin_amdgcn_readlane(weight, s0 + i));
        x += s0 + i < n_split ? v[i].x * w : 0.f;
        y += s0 + i < n_split ? v[i].y * w : 0.f;
      }
    }
    *reinterpret_cast<float2 *>(out + h * kHeadDim + 2 * lane) = make_float2(x, y);
  }
}

// The piece [tile0, tile1) of the row (b, kvh), whose tiles begin at row_at of the line; kAligned: the row's pieces and the block of its first.
struct DecPiece {
  int b, kvh, tile0, tile1, row_tiles, row_at, blk0, n_piece;
};

// Merges the waves' states (weighted sums o [G][d] each, a wave's at wave_floats; maxima and sums by head) behind a block barrier: into the output
// where the block has the entire row, else into the piece's slot, and the last block that finishes a piece of the row folds them.
template <bool kAligned, int kWaves>
__device__ __forceinline__ void finish_piece(const DecodeArgs &a, const float *o, int wave_floats, const float (&m)[kWaves][16], const float (&l)[kWaves][16],
                                             unsigned *last, DecPiece w) {
  constexpr int kThr = kWaves * 64;
  const int tid = threadIdx.x, G = a.G;
  const bool whole = w.tile0 == 0 && w.tile1 == w.row_tiles;
  float *part = a.part + (2 * (size_t)blockIdx.x + (!kAligned && w.tile0 == 0 ? 1 : 0)) * kDecodeSlotFloats;
  float *out = a.out + ((size_t)w.b * a.Hq + (size_t)w.kvh * G) * kHeadDim;
  for (int e = tid; e < G * (kHeadDim / 2); e += kThr) {
    const int h = e >> 6, d = (e & 63) * 2;
    float M = m[0][h];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) M = fmaxf(M, m[i][h]);
    float L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float f = dec_exp2(m[i][h] - M);
      const float2 ov = *reinterpret_cast<const float2 *>(o + i * wave_floats + h * kHeadDim + d);
      L += f * l[i][h];
      x += f * ov.x;
      y += f * ov.y;
    }
    if (whole) {
      const float sum = row_sum(L);
      *reinterpret_cast<float2 *>(out + h * kHeadDim + d) = make_float2(x / sum, y / sum);
    } else {
      agent_store2(part + h * kHeadDim + d, x, y);
      if (d == 0) agent_store2(part + kMaxReal * kHeadDim + 2 * h, M, L);
    }
  }
  if (whole) return;

  // ---- count this piece; the last one of the row folds them
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int blk0 = kAligned ? w.blk0 : dec_block_of(w.row_at, a.tiles, gridDim.x);
  const int n_split = kAligned ? w.n_piece : dec_block_of(w.row_at + w.row_tiles - 1, a.tiles, gridDim.x) - blk0 + 1;
  unsigned *count = a.count + (w.b * kMaxKvHeads + w.kvh) * kDecodeCountStride;
  if (tid == 0) {
    const unsigned old = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = old + 1u == (unsigned)n_split ? 1u : 0u;
  }
  __syncthreads();
  if (*last == 0u) return;
  if (tid == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next launch
  fold_row<kAligned, kWaves>(a, blk0, n_split, out);
}

}  // namespace fkv
