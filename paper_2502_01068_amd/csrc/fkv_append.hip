// New tokens' keys and values into a paged cache, rotary position embedding applied to the keys and queries on the way; and the
// writing side of the cache in 8 bits: appending to it, and KVCompress (App. B.1) into it.
//
// Rotation: (x, y) -> (x cos - y sin, y cos + x sin), phi = position * inv_freq[i].  Angles are held in turns as 64-bit whole numbers (2^64 = one
// turn): position * freq wraps around by itself, which reduces the angle exactly however far the position.  Its top 32 bits are
// used.  A block forms sine and cosine of its tokens once, in LDS, for all heads.
//
// A thread handles 16 columns of a row: two 16-byte chunks, which hold both columns of its 8 pairs (adjacent chunks, or chunks i and
// i + r/16 where pairs are half the turned columns apart); 8 threads make a row.
#include "fkv_quant.h"

namespace fkv {

constexpr int kRowLanes = 8;  // threads of a row
constexpr int kAppendMaxThreads = (kMaxKvHeads * kMaxReal + 2 * kMaxKvHeads) * kRowLanes;  // of a token
constexpr int kPairs = kHeadDim / 2;

// A launch's arguments where the hardware finds them.  (Through an ordinary reference, an index that differs between lanes, or a choice between
// two members, made the compiler copy all 1.6 KB to each lane's scratch memory first.)
typedef const __attribute__((address_space(4))) AppendArgs AppendKernArgs;
typedef const __attribute__((address_space(4))) QuantGatherArgs GatherKernArgs;
typedef const __attribute__((address_space(4))) int *kern_ints_t;
#define FKV_KERN_ARGS(type) (*(type *)__builtin_amdgcn_kernarg_segment_ptr())

// sine and cosine of a block's tokens, a row of kPairs each
template <int kTok>
struct TurnTable {
  float cs[kTok][kPairs], sn[kTok][kPairs];
};

// Sine and cosine of 2 pi t / 2^32.  The two top bits, rounded, are the quarter; what is left, a at most pi/4 in size, goes into Taylor's
// series, cut off where the next term is below 2^-28 (a^11 / 11!) and 2^-30 (a^12 / 12!).  Within 2^-23 in all.  Shorter than the library's
// sincospif: 64 tokens 4.6 -> 4.3 us.
__device__ __forceinline__ void turn_sincos(uint32_t t, float *sn, float *cs) {
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float a = (float)(int32_t)(t - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float w = a * a;
  float s = 1.f / 362880.f, c = -1.f / 3628800.f;
  s = fmaf(s, w, -1.f / 5040.f);
  s = fmaf(s, w, 1.f / 120.f);
  s = fmaf(s, w, -1.f / 6.f);
  s = fmaf(s * w, a, a);
  c = fmaf(c, w, 1.f / 40320.f);
  c = fmaf(c, w, -1.f / 720.f);
  c = fmaf(c, w, 1.f / 24.f);
  c = fmaf(c, w, -0.5f);
  c = fmaf(c, w, 1.f);
  const float x = quarter & 1 ? c : s, y = quarter & 1 ? s : c;  // a quarter on: sin -> cos, cos -> -sin
  *sn = __uint_as_float(__float_as_uint(x) ^ (quarter & 2) << 30);
  *cs = __uint_as_float(__float_as_uint(y) ^ ((quarter + 1) & 2) << 30);
}

// Rows 0 .. n - 1 of the table for the packed tokens token0, token0 + 1, ..: all threads of the block, a wave per token.  The frequency and the first
// positions are requested (constant memory: not in line with a thread's other loads) before the rest of the block's loads and used behind them.
template <int kTok>
struct TurnFill {
  static constexpr int kAhead = kTok < 8 ? kTok : 8;
  AppendKernArgs &a;
  int token0, n, i, wave, n_waves;
  uint64_t freq;
  int position[kAhead];

  __device__ __forceinline__ void request(int tok) {
    const auto positions = (kern_ints_t)a.positions;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) position[u] = positions[token0 + min(tok + u * n_waves, n - 1)];
  }
  __device__ __forceinline__ TurnFill(AppendKernArgs &args, int first, int count) : a(args), token0(first), n(count) {
    i = threadIdx.x & (kPairs - 1);
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kPairs);
    n_waves = blockDim.x / kPairs;
    freq = a.freq[min(i, max(a.pairs - 1, 0))];
    if (a.pairs > 0) request(wave);
  }
  __device__ __forceinline__ void fill(TurnTable<kTok> &t) {
    for (int tok = wave; tok < n; tok += kAhead * n_waves) {
      if (tok != wave) request(tok);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (tok + u * n_waves < n && i < a.pairs)
          turn_sincos((uint32_t)((uint64_t)(int64_t)position[u] * freq >> 32), &t.sn[tok + u * n_waves][i], &t.cs[tok + u * n_waves][i]);
    }
  }
};

// A block barrier that orders LDS only: a thread's loads in flight stay so.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where a thread's two chunks of a row lie; turned: they hold pairs 8 j .. 8 j + 7.
struct RowPart {
  int first, second;
  bool turned;
};
__device__ __forceinline__ RowPart row_part(AppendKernArgs &a, int j, bool rotate) {
  const int n_turn = a.pairs / 8;
  const bool turned = rotate && j < n_turn;
  return turned && !a.interleaved ? RowPart{j, j + n_turn, true} : RowPart{2 * j, 2 * j + 1, turned};
}

// The 16 values of a thread's chunks, turned by the pairs' angles.
__device__ __forceinline__ void turn16(AppendKernArgs &a, u32x4 first, u32x4 second, const float *cs, const float *sn, float (&x)[16]) {
  float v[16], c[8], s[8];
  unpack8(first, v);
  unpack8(second, v + 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = cs[i], s[i] = sn[i];
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * s[i];
      x[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = v[i] * c[i] - v[8 + i] * s[i];
      x[8 + i] = v[8 + i] * c[i] + v[i] * s[i];
    }
  }
}

// The sequence that entry i (uniform) of a packed batch belongs to: a prefix sum per lane, all of them in one load.
__device__ __forceinline__ int seq_at(kern_ints_t off, int n_seq, int i) {
  const int lane = threadIdx.x & 63;
  return __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n_seq - 1 && i >= off[min(lane, n_seq - 1) + 1]));
}

// The rows of kTok tokens: queries (n_q heads, into q_out), keys and values (n_kv heads each, into the pages).
template <int kTok>
__device__ __forceinline__ void append_rows(AppendKernArgs &a, TurnTable<kTok> &turns, int (&slots)[kTok], int token0, int n_q, int n_kv) {
  const int n_tok = min(kTok, a.total - token0), tid = threadIdx.x, j = tid & (kRowLanes - 1);
  const int rows_per = n_q + 2 * n_kv, n_rows = n_tok * rows_per;
  struct Row {
    int tok, h, kind;  // kind 0: query, 1: key, 2: value
    const u32x4 *src;
    RowPart part;
  };
  auto row_at = [&](int r) {
    Row w;
    w.tok = kTok == 1 ? 0 : r / rows_per;
    w.h = r - w.tok * rows_per;
    w.kind = w.h < n_q ? 0 : w.h < n_q + n_kv ? 1 : 2;
    w.h -= w.kind == 0 ? 0 : w.kind == 1 ? n_q : n_q + n_kv;
    const uint16_t *base = w.kind == 0 ? a.q : w.kind == 1 ? a.k : a.v;
    const int64_t stride = w.kind == 0 ? a.q_stride : w.kind == 1 ? a.k_stride : a.v_stride;
    w.src = reinterpret_cast<const u32x4 *>(base + (int64_t)(token0 + w.tok) * stride + w.h * kHeadDim);
    w.part = row_part(a, j, w.kind != 2);
    return w;
  };
  TurnFill<kTok> filler(a, token0, n_tok);
  // a thread's first row is on its way while angles and slots are looked up
  int r = tid / kRowLanes;
  Row w{};
  u32x4 first{}, second{};
  if (r < n_rows) {
    w = row_at(r);
    first = w.src[w.part.first];
    second = w.src[w.part.second];
  }
  if (n_kv > 0 && tid < 64) {  // the first wave, a lane per token
    int b = 0, at = 0;
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      const int token = min(token0 + i, a.total - 1), owner = seq_at(a.off, a.n_seq, token), place = a.start[owner] + token - a.off[owner];
      b = tid == i ? owner : b;
      at = tid == i ? place : at;
    }
    if (tid < n_tok) {
      const int page = a.block_table[(size_t)b * a.max_pages + (at >> a.page_shift)];
      slots[tid] = page >= 0 && page < a.n_pages ? (page << a.page_shift) + (at & ((1 << a.page_shift) - 1)) : -1;
    }
  }
  if (a.pairs > 0) filler.fill(turns);
  lds_barrier();
  for (bool more = false; r < n_rows; r += blockDim.x / kRowLanes, more = true) {
    if (more) {
      w = row_at(r);
      first = w.src[w.part.first];
      second = w.src[w.part.second];
    }
    if (w.part.turned) {
      float x[16];
      turn16(a, first, second, &turns.cs[w.tok][8 * j], &turns.sn[w.tok][8 * j], x);
      first = pack8(x);
      second = pack8(x + 8);
    }
    u32x4 *dst;
    if (w.kind == 0) {
      dst = reinterpret_cast<u32x4 *>(a.q_out + (int64_t)(token0 + w.tok) * a.q_out_stride + w.h * kHeadDim);
    } else {
      const int slot = slots[w.tok];
      if (slot < 0) continue;
      dst = reinterpret_cast<u32x4 *>((w.kind == 1 ? a.k_pages : a.v_pages) + ((size_t)slot * a.Hkv + w.h) * kHeadDim);
    }
    dst[w.part.first] = first;
    dst[w.part.second] = second;
  }
}

// A block takes one token, a thread 16 columns of one of its rows: nothing but the one memory trip behind the look-ups.  8191 tokens 37.2 us (5.4 TB/s; a large
// copy 5.2), 64 tokens 4.3; in a form that took longer to look up, 38.8 and 4.5, two tokens a block 41.8 and 5.7, four 43.1 and 8.2, eight 46.3 and 12.7.
__global__ __launch_bounds__(kAppendMaxThreads) void k_append(AppendArgs) {
  AppendKernArgs &a = FKV_KERN_ARGS(AppendKernArgs);
  __shared__ __attribute__((aligned(16))) TurnTable<1> turns;
  __shared__ int slots[1];
  append_rows<1>(a, turns, slots, blockIdx.x, a.q ? a.Hq : 0, a.Hkv);
}

// One scale block of one head, a wave's work: of its rows 0 .. kBlock - 1 (of kHeadDim bytes at `codes`) those of is_new are new, and
// earlier tokens lie in the `kept` rows at its begin.  A thread has row p * kRowLanes + lane / kRowLanes of step p, of which value(p, x) gives the
// 16 numbers of its two chunks.  No new row (a gather of negative indices): the smallest scale, so that none that memory held outlives it.
template <int kBlock, typename Value>
__device__ __forceinline__ void store_block(int kept, const bool (&is_new)[kBlock / kRowLanes], uint8_t *codes, float *scale, Value value, RowPart part) {
  constexpr int kSteps = kBlock / kRowLanes;
  const int lane = threadIdx.x & 63, sub = lane / kRowLanes;
  const float old = kept > 0 ? *scale : 0.f;
  float amax = 0.f;
  // The numbers are kept, in 64 registers at most, or formed again: 32 requests 6.2 against 6.6 us, keys and values of 11000 tokens 17.7 against 20.
  constexpr bool kKeep = kBlock <= 32;
  float x[kKeep ? kSteps : 1][16];
#pragma unroll
  for (int p = 0; p < kSteps; ++p) {
    if (is_new[p]) {
      float (&y)[16] = x[kKeep ? p : 0];
      value(p, y);
#pragma unroll
      for (int e = 0; e < 16; ++e) amax = fmaxf(amax, is_finite(y[e]) ? __builtin_fabsf(y[e]) : 0.f);
    }
  }
  amax = wave_fmax(amax);
  const float now = fmaxf(scale_for(amax), old), inv = 1.f / now;
  if (kept > 0 && now > old) {
    const float ratio = old / now;
    for (int i = lane; i < kept * 8; i += 64) {  // 16 codes each
      u32x4 *at = reinterpret_cast<u32x4 *>(codes) + i;
      u32x4 c = *at;
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = rescale4(c[e], ratio);
      *at = c;
    }
  }
#pragma unroll
  for (int p = 0; p < kSteps; ++p) {
    if (is_new[p]) {
      float (&y)[16] = x[kKeep ? p : 0];
      if constexpr (!kKeep) value(p, y);
      u32x2 *row = reinterpret_cast<u32x2 *>(codes + (p * kRowLanes + sub) * kHeadDim);
      const u32x2 first = encode8(y, inv), second = encode8(y + 8, inv);
      if (part.second == part.first + 1) {
        *reinterpret_cast<u32x4 *>(row + part.first) = u32x4{first[0], first[1], second[0], second[1]};
      } else {
        row[part.first] = first;
        row[part.second] = second;
      }
    }
  }
  if (lane == 0) *scale = now;
}

// Blocks of the grid: a scale block of a sequence for K, one for V (a wave for each head), and so on, then kAppendTok tokens' queries each (11000
// tokens, at 54.3 us now: 8 of them 61.5, 4 59.2, 2 57.2, 1 64.9, which leaves half of the threads idle).
constexpr int kAppendTok = 2;

template <int kBlock>
__global__ __launch_bounds__(kMaxKvHeads * 64) void k_append_quant(AppendArgs) {
  AppendKernArgs &a = FKV_KERN_ARGS(AppendKernArgs);
  constexpr int kTok = kBlock > kAppendTok ? kBlock : kAppendTok;
  __shared__ __attribute__((aligned(16))) TurnTable<kTok> turns;
  const int block = blockIdx.x, n_blk = 2 * a.blk[a.n_seq];
  if (block >= n_blk) {
    __shared__ int slots[kAppendTok];
    append_rows<kAppendTok>(a, reinterpret_cast<TurnTable<kAppendTok> &>(turns), slots, (block - n_blk) * kAppendTok, a.Hq, 0);
    return;
  }
  const bool is_v = (block & 1) != 0;
  const int at = block >> 1, b = seq_at(a.blk, a.n_seq, at);
  const int start = a.start[b], end = start + (a.off[b + 1] - a.off[b]);
  const int tok0 = (start / kBlock + (at - a.blk[b])) * kBlock;  // the block's first token
  const int first = max(start - tok0, 0), last = min(end - tok0, kBlock);
  const int token0 = a.off[b] + (tok0 + first - start);  // packed index of the first new token
  const int page = ((kern_ints_t)a.block_table)[(size_t)b * a.max_pages + (tok0 >> a.page_shift)];
  const bool turn = !is_v && a.pairs > 0;
  const int h = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & (kRowLanes - 1);
  const RowPart part = row_part(a, j, turn);
  TurnFill<kTok> filler(a, token0, last - first);
  // The rows are on their way while page and angles are looked up.
  const uint16_t *src = (is_v ? a.v : a.k) + h * kHeadDim;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  const int sub = lane / kRowLanes - first;  // of a thread's row among the new ones, in step 0
  u32x4 raw[kBlock / kRowLanes][2];
  bool is_new[kBlock / kRowLanes];
#pragma unroll
  for (int p = 0; p < kBlock / kRowLanes; ++p) {
    const int i = p * kRowLanes + sub;
    is_new[p] = i >= 0 && i < last - first;
    const u32x4 *r = reinterpret_cast<const u32x4 *>(src + (int64_t)(token0 + min(max(i, 0), last - first - 1)) * stride);
    raw[p][0] = r[part.first];
    raw[p][1] = r[part.second];
  }
  if (turn) {
    filler.fill(turns);
    lds_barrier();
  }
  if (page < 0 || page >= a.n_pages) return;
  const size_t row = (((size_t)page * a.Hkv + h) << a.page_shift) + (tok0 & ((1 << a.page_shift) - 1));
  store_block<kBlock>(
      first, is_new, (is_v ? a.v_codes : a.k_codes) + row * kHeadDim, (is_v ? a.v_scale : a.k_scale) + row / kBlock,
      [&](int p, float (&x)[16]) {
        if (part.turned) {
          const int i = p * kRowLanes + sub;
          turn16(a, raw[p][0], raw[p][1], &turns.cs[i][8 * j], &turns.sn[i][8 * j], x);
        } else {
          unpack8(raw[p][0], x);
          unpack8(raw[p][1], x + 8);
        }
      },
      part);
}

// KVCompress into the cache in 8 bits: a wave for a scale block of kept rows, of K or V and one head (heads fastest, then K and V).  Bound by bytes where
// there are many (13107 rows of 8 heads 18.1 us, 4.5 TB/s; all blocks are resident at once, so reading comes first and writing then), else by the
// chain indices - rows - maximum - codes (2048 rows 4.9).  Blocks of a wave for each head took 18.7 and 5.1 us, 16 threads to a row 19.8, non-temporal loads
// 21.4 (a thread's two loads share cache lines with its neighbours').
constexpr int kGatherWaves = 4;

template <int kBlock>
__global__ __launch_bounds__(kGatherWaves * 64) void k_gather_quant(QuantGatherArgs) {
  GatherKernArgs &a = FKV_KERN_ARGS(GatherKernArgs);
  constexpr int kSteps = kBlock / kRowLanes;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kGatherWaves + (threadIdx.x >> 6)), n_src = a.src[1] ? 2 : 1;
  const int line = (int)((uint32_t)unit / (uint32_t)a.Hkv), h = unit - line * a.Hkv;
  const int at = n_src == 2 ? line >> 1 : line, is_v = n_src == 2 ? line & 1 : 0;
  if (at >= a.blk[a.n_seq]) return;
  const int b = seq_at(a.blk, a.n_seq, at), lane = threadIdx.x & 63, j = lane & (kRowLanes - 1);
  const int tok0 = (at - a.blk[b]) * kBlock, last = min(a.cnt_off[b + 1] - a.cnt_off[b] - tok0, kBlock);
  const int page = ((kern_ints_t)a.block_table)[(size_t)b * a.max_pages + (tok0 >> a.page_shift)];
  const int all = a.idx[(size_t)h * a.total_rows + a.cnt_off[b] + tok0 + min(lane & (kBlock - 1), last - 1)];  // a lane each
  const int base = a.cu[b], n = a.cu[b + 1] - base;
  const uint16_t *src = a.src[is_v] + h * kHeadDim;
  u32x4 raw[kSteps][2];
  bool is_new[kSteps];
#pragma unroll
  for (int p = 0; p < kSteps; ++p) {
    const int i = p * kRowLanes + lane / kRowLanes, kept = __shfl(all, i);
    is_new[p] = i < last && kept >= 0;
    const u32x4 *r = reinterpret_cast<const u32x4 *>(src + (int64_t)(base + min(max(kept, 0), n - 1)) * a.Hkv * kHeadDim) + 2 * j;
    raw[p][0] = r[0];
    raw[p][1] = r[1];
  }
  if (page < 0 || page >= a.n_pages) return;
  const size_t row = (((size_t)page * a.Hkv + h) << a.page_shift) + (tok0 & ((1 << a.page_shift) - 1));
  store_block<kBlock>(
      0, is_new, a.codes[is_v] + row * kHeadDim, a.scale[is_v] + row / kBlock,
      [&](int p, float (&x)[16]) {
        unpack8(raw[p][0], x);
        unpack8(raw[p][1], x + 8);
      },
      RowPart{2 * j, 2 * j + 1, false});
}

hipError_t launch_append(const AppendArgs &a, hipStream_t s) {
  const int threads = (((a.q ? a.Hq : 0) + 2 * a.Hkv) * kRowLanes + 63) / 64 * 64;
  hipLaunchKernelGGL(k_append, dim3(a.total), dim3(threads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_append_quant(const AppendArgs &a, int block, hipStream_t s) {
  const dim3 grid(2 * a.blk[a.n_seq] + (a.q ? (a.total + kAppendTok - 1) / kAppendTok : 0)), threads(a.Hkv * 64);
  if (block == 16) hipLaunchKernelGGL((k_append_quant<16>), grid, threads, 0, s, a);
  else if (block == 32) hipLaunchKernelGGL((k_append_quant<32>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((k_append_quant<64>), grid, threads, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_gather_quant(const QuantGatherArgs &a, int block, hipStream_t s) {
  const int units = a.blk[a.n_seq] * a.Hkv * (a.src[1] ? 2 : 1);
  const dim3 grid((units + kGatherWaves - 1) / kGatherWaves), threads(kGatherWaves * 64);
  if (block == 16) hipLaunchKernelGGL((k_gather_quant<16>), grid, threads, 0, s, a);
  else if (block == 32) hipLaunchKernelGGL((k_gather_quant<32>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((k_gather_quant<64>), grid, threads, 0, s, a);
  return hipGetLastError();
}

}  // namespace fkv
