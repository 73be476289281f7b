// Decode-step attention over a paged cache held in 8 bits: out[h] = sum_t softmax_t(scale * q[h].k[g(h),t] ks_t) * v[g(h),t] vs_t, every
// cached token visible; k and v are e4m3 codes, ks and vs the scales of their blocks of tokens.
//
// Bound: the bytes of K and V, 256 per cached token and KV head.  As over a bf16 cache (fkv_decode.hip) both contractions run on the
// matrix cores in bf16, which holds every e4m3 value exactly; scales are applied in fp32, ks to the logits and vs to the probabilities.
//   S = K . Q^T    A operand = 16 tokens x 32 columns.  Lane (c, q) takes 16 bytes of token 8 (c / 4) + 4 h + c % 4 of the tile's 32, half h;
//                  they are 16 consecutive columns and feed two contraction steps (the queries are laid out to match).  The result
//                  leaves head c and the 8 consecutive tokens 8 q .. 8 q + 7 of the tile on a lane: one scale block.
//   O^T += V^T . P A operand = 16 columns x 32 tokens: a transposing LDS read (8 rows x 16 columns of bytes per 16 lanes) gives lane (c, q) column
//                  c of those same 8 tokens.  Probabilities enter as three bf16 pieces that add up to the fp32 value.
//
// A page holds a head's tokens one after the other, 128 bytes each, so a load instruction (64 lanes x 16 bytes) brings 8 whole
// tokens, of one page (pages have 16 or more).  All of it goes to wave-private LDS by LDS-direct loads, 16-byte columns swizzled on
// the global side by token and group of 8 so that neither read conflicts.  Two tiles of 32 tokens per wave are in flight (8.25 KB each with their
// scales), in two stages of LDS; waits count the loads behind the ones that are needed (in asm: for ordinary LDS reads the
// compiler would wait for all).  Page entries come 32 tiles at a time, a lane each.
//
// Work is spread and rows folded as in fkv_decode.hip.
//
// Measured (kernel time, us): one sequence of 32 tokens 4.8, 2048 7.0, 8192 10.0, 32768 17.8, 131072 47.2 (5.7 TB/s; 6.9 from 65536 tokens to there, the
// card's rate for reads); 32 sequences of 2048-2560 29.0 (5.3 TB/s).  A wave has a tile's work done in 1.0 us, two waves of a SIMD in 1.4; the bytes of a
// CU's 8 tiles take 2.4.  One wait for K and V together was slower (32768 tokens 19.0: K's contraction then waits for V).
#include <algorithm>
#include <type_traits>

#include "fkv_decode_common.h"
#include "fkv_quant.h"

namespace fkv {

constexpr int kTileBytes = kDecTile * kHeadDim;          // of K or V
constexpr int kStageBytes = 2 * kTileBytes + 256;        // K, V, scales (K's two at 0 and 64, V's at 128 and 192)
constexpr int kStages = 2;

__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {  // 8 codes as bf16
  struct { bf16x2 v[4]; } r = {{__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                                __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)}};
  return __builtin_bit_cast(bf16x8, r);
}

// The K tile's operands (halves of 16 tokens, then the 16-byte columns q and q + 4) and the scales of a lane's 8 tokens, once all but the
// kYounger youngest loads are there; returns when they are read, so that the tile may be overwritten.
template <int kYounger>
__device__ __forceinline__ void read_k(u32x4 (&r)[4], float &ks, float &vs, uint32_t addr, uint32_t scale_addr) {
  asm volatile(
      "s_waitcnt vmcnt(%8)\n\t"
      "ds_read_b128 %0, %6\n\t"
      "ds_read_b128 %1, %6 offset:64\n\t"
      "ds_read_b128 %2, %6 offset:576\n\t"
      "ds_read_b128 %3, %6 offset:512\n\t"
      "ds_read_b32 %4, %7\n\t"
      "ds_read_b32 %5, %7 offset:128\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(ks), "=&v"(vs)
      : "v"(addr), "v"(scale_addr), "n"(kYounger)
      : "memory");
}

// The V tile, transposed: r[j] holds column 16 j + c of a lane's 8 tokens.
template <int kYounger>
__device__ __forceinline__ void read_v(u32x2 (&r)[8], const uint32_t (&addr)[8]) {
  asm volatile(
      "s_waitcnt vmcnt(%16)\n\t"
      "ds_read_b64_tr_b8 %0, %8\n\t"
      "ds_read_b64_tr_b8 %1, %9\n\t"
      "ds_read_b64_tr_b8 %2, %10\n\t"
      "ds_read_b64_tr_b8 %3, %11\n\t"
      "ds_read_b64_tr_b8 %4, %12\n\t"
      "ds_read_b64_tr_b8 %5, %13\n\t"
      "ds_read_b64_tr_b8 %6, %14\n\t"
      "ds_read_b64_tr_b8 %7, %15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]), "v"(addr[4]), "v"(addr[5]), "v"(addr[6]), "v"(addr[7]), "n"(kYounger)
      : "memory");
}

// A lane's four operands from the queries in LDS: head c, columns 16 (q + 4 u) + 8 e .. + 7 in step 2 u + e.
template <int kYounger>
__device__ __forceinline__ void read_q(bf16x8 (&qb)[4], uint32_t addr, bool live) {
  u32x4 r[4];
  asm volatile(
      "s_waitcnt vmcnt(%5)\n\t"
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %4 offset:16\n\t"
      "ds_read_b128 %2, %4 offset:128\n\t"
      "ds_read_b128 %3, %4 offset:144\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(addr), "n"(kYounger)
      : "memory");
#pragma unroll
  for (int s = 0; s < 4; ++s) qb[s] = __builtin_bit_cast(bf16x8, live ? r[s] : u32x4{0u, 0u, 0u, 0u});
}

template <bool kAligned, int kWaves>
__global__ __launch_bounds__(kWaves * 64, 2) void k_decode_quant(DecodeQuantArgs args) {
  const DecodeArgs &a = args.d;
  __shared__ __attribute__((aligned(256))) uint8_t stage_lds[kWaves][kStages * kStageBytes];
  __shared__ __attribute__((aligned(16))) uint8_t q_lds[kWaves][kMaxReal * kHeadDim * 2];
  __shared__ float m_lds[kWaves][16], l_lds[kWaves][16];
  __shared__ unsigned last_lds;
  typedef __attribute__((address_space(1))) const void *gptr_t;
  typedef __attribute__((address_space(1))) const uint8_t *rows_t;
  typedef __attribute__((address_space(3))) void *lptr_t;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int G = a.G;
  int b = 0, at, at_end;
  int n_piece = 1, piece_blk0 = 0, kvh0 = 0;  // kAligned: pieces of the row, the block of its first one, its KV head
  if (kAligned) {
    const int unit = (int)((uint32_t)blockIdx.x / (uint32_t)a.Hkv);  // pieces before this one, KV heads left aside
    for (int i = 1; i < a.n_seq && b == i - 1; i += 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) b += (i + j < a.n_seq) & (unit >= a.piece0[i + j]);
    }
    n_piece = a.piece0[b + 1] - a.piece0[b];
    const int p = unit - a.piece0[b];
    kvh0 = (int)blockIdx.x - unit * a.Hkv;
    piece_blk0 = (int)blockIdx.x - p * a.Hkv;
    const int len = a.tile0[b + 1] - a.tile0[b];
    at = 0;
    at_end = len;
    if (n_piece > 1) {
      at = (int)share_at(len, p, n_piece);
      at_end = (int)share_at(len, p + 1, n_piece);
    }
  } else {
    at = (int)share_at(a.tiles, blockIdx.x, gridDim.x);
    at_end = (int)share_at(a.tiles, blockIdx.x + 1, gridDim.x);
  }
  uint8_t *stage = stage_lds[wave];
  const uint32_t stage_addr = (uint32_t)(uintptr_t)(lptr_t)stage;
  // 16-byte column u of token t lies at column u ^ (t % 8) ^ (t / 8) of its row in LDS.
  const int k_tok = 8 * (c >> 2) + (c & 3);  // of half 0; half 1: 4 tokens on, in which the swizzle flips column bit 2, as q + 4 does
  const uint32_t k_at = k_tok * kHeadDim + ((q ^ (c & 3) ^ (c >> 2)) << 4);
  const int v_row = c >> 1;
  const uint32_t v_at = kTileBytes + (8 * q + v_row) * kHeadDim + ((v_row ^ q) << 4) + 8 * (c & 1);
  const uint32_t load_at = (lane >> 3) * kHeadDim + (((lane & 7) ^ (lane >> 3)) << 4);  // of a load's 8 tokens; ^ 16 i for tokens 8 i ..

  while (at < at_end) {
    // ---- the piece [tile0, tile1) of row (b, kvh)
    int row_at = 0, kvh = kvh0;  // kAligned: `at` counts from the row's first tile
    if (!kAligned) {
      while (at >= a.tile0[b + 1] * a.Hkv) ++b;
    }
    const int row_tiles = a.tile0[b + 1] - a.tile0[b];
    if (!kAligned) {
      const int seq_at = a.tile0[b] * a.Hkv;
      kvh = (int)((uint32_t)(at - seq_at) / (uint32_t)row_tiles);
      row_at = seq_at + kvh * row_tiles;
    }
    const int tile0 = at - row_at, tile1 = min(row_tiles, at_end - row_at);
    at = row_at + tile1;
    const int n = a.off[b + 1] - a.off[b];
    if (n == 0) {  // no token: zeros
      for (int e = tid; e < G * kHeadDim; e += kWaves * 64) a.out[((size_t)b * a.Hq + (size_t)kvh * G) * kHeadDim + e] = 0.f;
      if (kAligned) return;
      continue;
    }

    const int32_t *table = a.block_table + (size_t)b * a.max_pages;
    const int last_page = (n - 1) >> a.page_shift;
    // Page entries of 32 of the wave's tiles, from its `first`-th on: lane l has that of half l % 2 of tile l / 2; clamped into the pool.
    auto page_batch = [&](int first) {
      const int t = min(tile0 + wave + (first + (lane >> 1)) * kWaves, tile1 - 1) * kDecTile + 16 * (lane & 1);
      return min(max(table[min(t >> a.page_shift, last_page)], 0), a.n_pages - 1);
    };
    const int in_page = (1 << a.page_shift) - 1;
    int pages = 0;
    // Requests the wave's i-th tile into its stage: scales and K, then V, in that order.
    struct Place {
      uint32_t row[2];  // of either half's first token: page, head and slot, in tokens
    };
    auto place_of = [&](int i) {
      Place p;
      const int t = (tile0 + wave + i * kWaves) * kDecTile;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages, 2 * (i & 31) + h);
        p.row[h] = ((page * (uint32_t)a.Hkv + kvh) << a.page_shift) + ((t + 16 * h) & in_page);
      }
      return p;
    };
    auto load_tile = [&](rows_t base, const Place &p, int i, int offset) {
      uint8_t *to = stage + (i & 1) * kStageBytes + offset;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        rows_t rows = base + ((uint64_t)p.row[g >> 1] << 7) + (g & 1) * 1024;
        __builtin_amdgcn_global_load_lds((gptr_t)(rows + (load_at ^ (g << 4))), (lptr_t)(to + g * 1024), 16, 0, 2);
      }
    };
    auto load_k = [&](const Place &p, int i) {
      const float *scales = lane < 32 ? args.k_scale : args.v_scale;
      __builtin_amdgcn_global_load_lds((gptr_t)(scales + ((lane & 16 ? p.row[1] : p.row[0]) >> args.block_shift)),
                                       (lptr_t)(stage + (i & 1) * kStageBytes + 2 * kTileBytes), 4, 0, 0);
      load_tile((rows_t)args.k, p, i, 0);
      keep_access_order();
    };
    auto load_v = [&](const Place &p, int i) {
      load_tile((rows_t)args.v, p, i, kTileBytes);
      keep_access_order();
    };

    bf16x8 qb[4];
    floatx4 o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    float m = kDecNegBig, l = 0.f;

    // One tile; kAhead: how many of the wave's next ones there are (0, 1, or 2 or more; the second one is requested here as its stage becomes
    // free).  Loads behind K's: V's 4, and 9 of the next tile; behind V's: those 9, and 5 of the one after.
    auto step = [&](int i, auto ahead_t) {
      constexpr int kAhead = decltype(ahead_t)::value;
      const uint32_t from = stage_addr + (i & 1) * kStageBytes;
      u32x4 kr[4];
      float ks, vs;
      read_k<kAhead ? 13 : 4>(kr, ks, vs, from + k_at, from + 2 * kTileBytes + (q >> 1) * 64);
      Place next;
      if constexpr (kAhead == 2) {
        next = place_of(i + 2);
        load_k(next, i + 2);
      }
      floatx4 acc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        acc[h] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x4 k = kr[2 * h + u];
          acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(k[0], k[1]), qb[2 * u], acc[h], 0, 0, 0);
          acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(k[2], k[3]), qb[2 * u + 1], acc[h], 0, 0, 0);
        }
      }

      // acc[h][r] = logit of head c and token 8 q + 4 h + r of the tile, without its scale
      const int left = n - ((tile0 + wave + i * kWaves) * kDecTile + 8 * q);  // of a lane's 8 tokens these many count
      const bool edge = (tile0 + wave + i * kWaves + 1) * kDecTile > n;
      float z[8];
      float tmax = kDecNegBig;
      const float kscale = ks * a.scale_log2e;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = acc[e >> 2][e & 3] * kscale;
        if (edge && e >= left) z[e] = -INFINITY;  // weight 0 below whatever the maximum: it is at least kDecNegBig
        tmax = fmaxf(tmax, z[e]);
      }
      tmax = quarters_max(tmax);
      const float m_new = fmaxf(m, tmax);
      const float alpha = dec_exp2(m - m_new);
      m = m_new;
      float psum = 0.f;
      // p vs = p0 + p1 + p2, 8 bits each, cut off and not rounded
      if (edge) vs = left > 0 ? vs : 0.f;  // of a block that no token is in
      u32x4 p0, p1, p2;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        uint32_t w0[2], w1[2], w2[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float p = dec_exp2(z[e + s] - m_new);
          psum += p;
          const float pv = p * vs;
          w0[s] = __float_as_uint(pv);
          const float r1 = pv - __uint_as_float(w0[s] & 0xffff0000u);
          w1[s] = __float_as_uint(r1);
          w2[s] = __float_as_uint(r1 - __uint_as_float(w1[s] & 0xffff0000u));
        }
        p0[e / 2] = __builtin_amdgcn_perm(w0[1], w0[0], 0x07060302u);
        p1[e / 2] = __builtin_amdgcn_perm(w1[1], w1[0], 0x07060302u);
        p2[e / 2] = __builtin_amdgcn_perm(w2[1], w2[0], 0x07060302u);
      }
      l = l * alpha + psum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] *= alpha;
      }

      u32x2 va[8];
      uint32_t v_addr[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v_addr[j] = from + (v_at ^ (j << 4));
      read_v<(kAhead ? 9 : 0) + (kAhead == 2 ? 5 : 0)>(va, v_addr);
      if constexpr (kAhead == 2) load_v(next, i + 2);
      if (edge) {  // what lies behind the sequence may be NaN, which times 0 would stay
        const uint64_t mask = left >= 8 ? ~0ull : left <= 0 ? 0ull : (1ull << (8 * left)) - 1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          va[j][0] &= (uint32_t)mask;
          va[j][1] &= (uint32_t)(mask >> 32);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bf16x8 vj = widen(va[j][0], va[j][1]);
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vj, __builtin_bit_cast(bf16x8, p2), o[j], 0, 0, 0);
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vj, __builtin_bit_cast(bf16x8, p1), o[j], 0, 0, 0);
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vj, __builtin_bit_cast(bf16x8, p0), o[j], 0, 0, 0);
      }
    };

    const int mine = (tile1 - tile0 - wave + kWaves - 1) / kWaves;  // the wave's tiles (0 or less: none)
    if (mine > 0) {
      pages = page_batch(0);
      const auto rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.q + ((size_t)b * a.Hq + (size_t)kvh * G) * kHeadDim), 0,
                                                          G * kHeadDim * 2, 0x00027000);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lptr_t)(q_lds[wave] + i * 1024), 16, i * 1024 + lane * 16, 0, 0, 0);
      keep_access_order();
      const Place first = place_of(0);
      load_k(first, 0);
      load_v(first, 0);
      const uint32_t q_addr = (uint32_t)(uintptr_t)(lptr_t)q_lds[wave] + (c & 7) * 256 + q * 32;
      if (mine > 1) {
        const Place second = place_of(1);
        load_k(second, 1);
        load_v(second, 1);
        read_q<18>(qb, q_addr, c < G);
      } else {
        read_q<9>(qb, q_addr, c < G);
      }
      int i = 0;
      for (; i + 2 < mine; ++i) {
        if (((i + 2) & 31) == 0) pages = page_batch(i + 2);
        step(i, std::integral_constant<int, 2>{});
      }
      if (i + 1 < mine) step(i++, std::integral_constant<int, 1>{});
      step(i, std::integral_constant<int, 0>{});
    }

    // ---- the waves' states into LDS, in place of their tiles: lane (head c, q) holds d = 16 j + 4 q + r in o[j][r]
    l = quarters_sum(l);
    float *o_lds = reinterpret_cast<float *>(stage);
    if (c < G) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<float4 *>(o_lds + c * kHeadDim + 16 * j + 4 * q) = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
      if (q == 0) { m_lds[wave][c] = m; l_lds[wave][c] = l; }
    }
    __syncthreads();
    finish_piece<kAligned, kWaves>(a, reinterpret_cast<float *>(stage_lds[0]), kStages * kStageBytes / (int)sizeof(float), m_lds, l_lds, &last_lds,
                                   DecPiece{b, kvh, tile0, tile1, row_tiles, row_at, piece_blk0, n_piece});
    if (kAligned) return;
    __syncthreads();
  }
}

hipError_t launch_decode_quant(DecodeQuantArgs &a, int n_cu, hipStream_t s) {
  // Blocks of 8 waves, one to a CU (149 KB of LDS); of 4
  //   where there are more rows than CUs, two to a CU, so that one block's start is covered by the other.  us, 8 waves and 4: 256 rows of 2048-2560
  //   tokens 29.3, 30.6; one sequence of 131072 (8 rows) 47.1, 49.0; 128 rows of 1000 12.5, 12.3; but 512 rows of 2000 50.3, 45.4; of 200 13.5, 9.9;
  //   384 rows of 500-1000 25.2, 23.0; 264 of 600-1200 21.1, 17.5;
  //   where a tile for each wave leaves half of the CUs idle: the SIMDs then have one wave each.  One sequence of 1024 tokens 7.9, 7.3, 2048 7.9,
  //   7.3; 3000 8.0, 8.3.  Not where rows stay whole: 512 7.2, 7.5.
  const int rows = a.d.n_seq * a.d.Hkv;
  int64_t tiles = 0, longest = 0;
  for (int b = 0; b < a.d.n_seq; ++b) {
    const int64_t t = (a.d.off[b + 1] - a.d.off[b] + kDecTile - 1) / kDecTile;
    tiles += t * a.d.Hkv;
    longest = std::max(longest, t);
  }
  const bool few = tiles <= 2 * n_cu && longest > kDecQuantWhole, wide = rows <= n_cu && !few;
  const DecodePlan plan = wide ? plan_decode(a.d, n_cu, 8, true) : plan_decode(a.d, few ? n_cu : 2 * n_cu, 4, true);
  auto launch = [&](auto aligned_t, auto waves_t) {
    constexpr int kWaves = decltype(waves_t)::value;
    hipLaunchKernelGGL((k_decode_quant<decltype(aligned_t)::value, kWaves>), dim3(plan.blocks), dim3(kWaves * 64), 0, s, a);
  };
  using four = std::integral_constant<int, 4>;
  using eight = std::integral_constant<int, 8>;
  if (plan.aligned) wide ? launch(std::true_type{}, eight{}) : launch(std::true_type{}, four{});
  else wide ? launch(std::false_type{}, eight{}) : launch(std::false_type{}, four{});
  return hipGetLastError();
}

}  // namespace fkv
