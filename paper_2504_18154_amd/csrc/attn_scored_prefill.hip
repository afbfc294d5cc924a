// Attention of prompts (chunks of them, behind what is cached) over the caches of ecoserve_cache, with formed scores, on gfx950 matrix cores.
//
// Eq. 2 of Section 2.1 for the prefill phase, bound by the matrix units and the vector work of the softmax beside them.  A tile is 128 or 256 rows ((position,
// query head of the group) pairs of one sequence and K/V head), 32 to each of four or eight wavefronts, which share the tile's keys, 64 at a time:
//   scores  S^T[key][row] = K . Q^T     v_mfma_f32_32x32x16_bf16
//   values  O^T[d][row] += V^T . P^T    v_mfma_f32_32x32x16_bf16
// A step's codes are loaded two steps ahead, and a step ahead turned into bf16, scales and all (exact: a code has 7 bits at most and the scales are powers
// of two), on the way into LDS, once for the tile's wavefronts; the loop over the keys is the same for all formats.
//   K in LDS: [16-byte unit of 8 channels][64 keys], V: [8 keys][channel][16 bytes]; both are read as A operands, 16 bytes a lane.
// Rows of S^T stand for keys with bits 2 and 3 swapped, so that the 16 scores that a lane holds of 32 keys are two runs of 8 neighbouring keys: the B
// operand of the second product, and P stays in registers.
//
// A row's keys are a range.  The tile walks the steps from the first range's begin to the last range's end; a wavefront passes over steps that none of its
// rows sees, and masks only where a step is not inside all its rows' ranges.  Ranges that are given may leave keys between them that no row of the tile sees: tiles where
// neighbouring rows' ranges do not touch look at each step for the keys that are seen, from all rows' ranges in LDS; other keys' blocks are not named, and their values zeros.
// Tiles are dealt heaviest first.  Where they are few, their steps are cut among several workgroups; each leaves its state in the workspace, and the last
// one to arrive adds them up in order.
//
// Values that are not finite must not reach rows that do not see them (0 times NaN).  Codes: such a row is coded as zeros, its scale byte says 255, and rows that
// see it are given NaN at the end.  bf16: where a result is not finite and a key that the row does not see may be why, it is taken again over those that it sees.
//
// Weights are rounded to bf16 for the second product (2^-9 of each, unbiased) where the cache's codes, of 4 and 7 bits, are coarser, and in heads of 128, as in the other call for prompts of
// those; over bf16 caches of other heads, where that call holds more, they are two bf16 numbers, 16 bits, and products of their own (us with one part and with two: 4 x 4096 tokens, 8 heads on 1 of
// 256 over bf16 389 and 475, 8 on 8 of 80 163 and 204;  what was not taken: over e4m3 446 and 557, two of 8192, 64 heads on 8 of 128 2190 and 2990).  Maxima, sums and the log-sum-exp are
// fp32, from the weights as they were.
//
// Measured, 64 heads on 8 of 128: two prompts of 8192 tokens over e4m3 2100 ... 2190 us from card to card (1045 ... 1005 TFLOP/s; a library product of 8192^3 reaches 1220), over bf16
// 2040 ... 2145; a step of 64 keys is 201 vector instructions beside 32 matrix ones of a wavefront, the units are busy 47 and 45% of the time, LDS has no bank conflicts, and the clock gives
// way: fewer instructions raise it more than they save cycles.  Capped scores cost four vector instructions each, two of them at half rate (2048 tokens of three
// prompts 129 us).  24 prompts of 5 ... 300 tokens, 32 heads on 8 of 64, biased: 23.4 us, of which 5 are a workgroup's way to its first keys.
//
// Lane layouts relied upon (lane = 32 half + col), 32x32x16:  A[row = col][k = 8 half .. + 7],  B[k = 8 half .. + 7][col],
// C[row = 8 (i / 4) + 4 half + i % 4][col].
#include <type_traits>

#include "quant.h"
#include "scored.h"
#include "softcap.h"

namespace eco {

namespace {

constexpr int kKeys = 64;
constexpr float kLowest = -3.0e38f;  // maximum before the first key: below every finite score, and no infinity to be subtracted from one
// The offset in the exponent is put this far above the largest score (log2 units), and again when one passes it: no weight is above 1, so that no sum leaves fp32 for the offset,
// and weights lose nothing by being small.
constexpr float kRoom = 8.f;
constexpr int kRsrc = 0x00020000;
constexpr int kAgent = 16;           // past the caches that XCDs do not share

__device__ __forceinline__ float across_halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float across_halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <int F, int NC, bool kFull, int kWaves>
struct Tile {
  static constexpr int kThreads = 64 * kWaves, kRows = 32 * kWaves;  // of a workgroup
  static constexpr bool kNarrow = F != kNative;
  static constexpr bool kTwo = !kNarrow && !(NC == 4 && kFull);     // weights in two parts
  static constexpr int kD = 32 * NC;                                // channels that the instance holds
  static constexpr int kUnits = kD / 8;                             // of 8 channels
  static constexpr int kKBytes = kUnits * kKeys * 16;
  static constexpr int kOctet = kD * 16 + 64;                       // 8 keys of V, and what moves the next ones to other banks
  static constexpr int kVBytes = 8 * kOctet;
  static constexpr int kBuffers = NC == 8 ? 1 : 2;                  // (heads of 256: a second one would leave a workgroup per CU)
  static constexpr int kChunks = (kNarrow ? 2 : 4) * NC / kWaves;   // 16-byte loads of K, and of V, per thread and step
};

// The tile that `rank` others come before, by falling length (the keys that its last row sees, in at most 16 classes), in a batch of up to 64 sequences, one to a
// lane; b = -1 behind the last tile.  A sequence's tiles grow longer, so those of class v and above are its last ones, and their number is a formula: v is found by
// halving.  24 prompts of 5 ... 300 tokens: 30.4 us in the sequences' order, 26.6 in this one, which costs a workgroup 0.7 us (two prompts of 8192 tokens, which it
// has nothing to offer: 2242 and 2265; all with tiles of 128 rows).  Where ranges are given the lengths are not known: three prompts of several documents 147 and 162.
struct TileOf {
  SeqOf seq;
  int tile;
};
template <int kRows>
__device__ __forceinline__ TileOf heaviest_tile(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ ctx_before, int B, int G, int rank) {
  const int b = min((int)(threadIdx.x & 63), B - 1);
  const int tok0 = cu_q[b], S = (int)(threadIdx.x & 63) < B ? cu_q[b + 1] - tok0 : 0, cb = ctx_before[b];
  const int tiles = S > 0 ? (S * G + kRows - 1) / kRows : 0;
  const int steps = lanes_max(tiles && cb + S > 0 ? (cb + S - 1) / kKeys + 1 : 0), shift = max(0, 28 - __builtin_clz(steps | 1));
  // the first tile of class v: its last row sees key (v - 1) 64 2^shift
  auto first_of = [&](int v) {
    const long long at = ((long long)kKeys << shift) * (v - 1) - cb;
    return v <= 0 || at <= 0 ? 0 : at >= S ? tiles : (int)at * G / kRows;
  };
  auto add = [](int x, int y) { return x + y; };
  int lo = 0, hi = ((steps + (1 << shift) - 1) >> shift) + 1, above = 0;
  while (hi - lo > 1) {
    const int v = (lo + hi) >> 1, n = __builtin_amdgcn_readlane(lanes_scan(tiles - first_of(v), add), 63);
    if (n > rank) lo = v;
    else hi = v, above = n;
  }
  // (the rank's class is lo, and `above` tiles have higher ones)
  const int upto = lanes_scan(first_of(hi) - first_of(lo), add);
  const unsigned long long reach = __ballot(upto > rank - above);
  TileOf r;
  r.seq.b = -1;
  if (!reach) return r;
  const int who = __builtin_ctzll(reach);
  r.seq.b = who;
  r.seq.tok0 = __builtin_amdgcn_readlane(tok0, who);
  r.seq.S = __builtin_amdgcn_readlane(S, who);
  r.seq.cb = __builtin_amdgcn_readlane(cb, who);
  r.tile = __builtin_amdgcn_readlane(first_of(hi), who) - (__builtin_amdgcn_readlane(upto, who) - (rank - above));
  return r;
}

enum { kPlain, kCapped, kBiased, kFarCapped };  // scores: scaled, capped (near: softcap.h), with a bias (capped or not), or capped far above them, with a bias or without

// What a row of scores needs of the score's form.
struct Form {
  Cap cap;
  float by, start;  // without a bias: scores are by s + start, s the products or what their caps make of them
  const float* slopes;
};

// Keys k0 .. k0 + 63 that one of n rows sees (n a multiple of 64).
__device__ __forceinline__ uint64_t seen_by_rows(const int* row_lo, const int* row_hi, int n, int k0) {
  uint64_t m = 0;
  for (int r = threadIdx.x & 63; r < n; r += 64) m |= keys_seen(row_lo[r], row_hi[r], k0);
  uint32_t a = (uint32_t)m, b = (uint32_t)(m >> 32);
#pragma unroll
  for (int w = 1; w < 64; w *= 2) a |= (uint32_t)__shfl_xor((int)a, w), b |= (uint32_t)__shfl_xor((int)b, w);
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)b) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)a);
}

// Whether a value of keys [from, to) is not finite.  (n > 0: of those that one of the n rows sees.)
__device__ __attribute__((noinline)) bool not_finite_in(const char* __restrict__ v_head, uint32_t blk_stride, const int32_t* __restrict__ table, int from, int to, int D,
                                                        const int* row_lo, const int* row_hi, int n) {
  bool odd = false;
  for (int blk = from >> 4; blk * kBlockSize < to; ++blk) {
    const uint32_t slots = n ? (uint32_t)seen_by_rows(row_lo, row_hi, n, blk * kBlockSize) & 0xffffu : 0xffffu;
    if (!slots) continue;
    const char* const at = v_head + (size_t)(uint32_t)table[blk] * blk_stride;
    for (int u = threadIdx.x & 63; u < 2 * D; u += 64) {  // (half of a channel's slots)
      const u32x4 x = *reinterpret_cast<const u32x4*>(at + u * 16);
      const int key = blk * kBlockSize + 8 * (u & 1);
#pragma unroll
      for (int e = 0; e < 8; ++e) odd |= key + e >= from && key + e < to && (slots >> (8 * (u & 1) + e) & 1) && (x[e >> 1] >> (16 * (e & 1)) & 0x7f80u) == 0x7f80u;
    }
  }
  return __any(odd);
}

// One row again, from its keys alone, by a wavefront: lane l has channels l, l + 64, ...  For results that are not finite, where a value that the row does not
// see may be the cause.
template <int NC, int kForm>
__device__ __attribute__((noinline)) void row_again(const uint16_t* __restrict__ q_row, const char* __restrict__ k_head, const char* __restrict__ v_head, long long blk_stride,
                                                    const int32_t* __restrict__ table, int lo, int hi, int pos, float slope, Form form, int D, uint16_t* __restrict__ to) {
  constexpr int kPer = NC == 8 ? 4 : NC == 4 ? 2 : 1;
  const int lane = threadIdx.x & 63;
  float qv[kPer], o[kPer], m = kLowest, l = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int d = lane + 64 * i;
    qv[i] = d < D ? bf16_bits_to_float(q_row[d]) : 0.f;
    o[i] = 0.f;
  }
  for (int j = lo; j < hi; ++j) {
    const long long at = (long long)table[j >> 4] * blk_stride;
    const uint16_t *const kp = reinterpret_cast<const uint16_t*>(k_head + at), *const vp = reinterpret_cast<const uint16_t*>(v_head + at);
    float s = 0.f, v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = min(lane + 64 * i, D - 1);
      s += lane + 64 * i < D ? qv[i] * bf16_bits_to_float(kp[(d >> 3) * 128 + (j & 15) * 8 + (d & 7)]) : 0.f;
      v[i] = bf16_bits_to_float(vp[d * 16 + (j & 15)]);
    }
    s = wave_sum(s);
    if (kForm == kFarCapped) s = far_cap(s, form.cap);
    else s = __builtin_fmaf(kForm != kPlain && form.cap.kind == kNear ? near_cap(s, form.cap) : s, form.by, form.start);
    if (kForm == kBiased || kForm == kFarCapped) s = __builtin_fmaf(slope, (float)(j - pos), s);
    const float m_new = fmaxf(m, s), alpha = __builtin_amdgcn_exp2f(m - m_new), p = __builtin_amdgcn_exp2f(s - m_new);
    l = l * alpha + p;
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = o[i] * alpha + p * v[i];
    m = m_new;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (const int d = lane + 64 * i; d < D) to[d] = float_to_bf16_bits(o[i] / l);
}

// Workgroup (x, y): K/V head x % Hkv of tile x / Hkv, counted from the last one; y: which part of its steps.
// kFull: the head vector fills the instance's channels.
template <int F, int NC, int kForm, bool kFull, int kWaves>
__global__ __launch_bounds__(64 * kWaves, NC == 8 ? 1 : 2) void prefill_scored_kernel(
    const uint16_t* __restrict__ q, int q_row_stride, const char* __restrict__ k_cache, const char* __restrict__ v_cache, const uint8_t* __restrict__ scales,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ ctx_before, const int32_t* __restrict__ block_table, int bt_stride,
    const int32_t* __restrict__ key_begin, const int32_t* __restrict__ key_end, uint16_t* __restrict__ out, float* __restrict__ lse, float* states,
    uint32_t* counters, int B, int Hq, int Hkv, int G, Divisor div_g, Divisor div_hkv, int D, int units, Form form) {
  typedef Cached<F> C;
  typedef Tile<F, NC, kFull, kWaves> W;
  __shared__ __attribute__((aligned(16))) char s_k[W::kBuffers][W::kKBytes], s_v[W::kBuffers][W::kVBytes];
  __shared__ int s_lo[kWaves], s_hi[kWaves], s_order, s_bad[2], s_row_lo[W::kRows], s_row_hi[W::kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;

  // ---- the tile, its rows and their keys
  const int xu = fast_div((int)blockIdx.x, div_hkv), g = (int)blockIdx.x - xu * Hkv, unit = units - 1 - xu;
  auto first_unit = [&](int cu, int b) { return (long long)prefill_scored_first_tile(W::kRows, G, cu, b); };
  TileOf at_tile;
  if (B > 2 && B <= 64 && !key_begin && !key_end) {
    at_tile = heaviest_tile<W::kRows>(cu_q, ctx_before, B, G, xu);
    if (at_tile.seq.b < 0) return;
  } else {
    at_tile.seq = find_sequence(cu_q, ctx_before, B, unit, first_unit);
    at_tile.tile = (int)(unit - first_unit(at_tile.seq.tok0, at_tile.seq.b));
  }
  const SeqOf seq = at_tile.seq;
  const int rows = seq.S * G, row0 = at_tile.tile * W::kRows;
  if (seq.S <= 0 || row0 >= rows) return;
  const int rr = row0 + wave * 32 + col, place = fast_div(min(rr, rows - 1), div_g), head = g * G + min(rr, rows - 1) - place * G, tok = seq.tok0 + place;
  const bool valid = rr < rows;
  const int pos = seq.cb + place, total = seq.cb + seq.S;
  int lo = key_begin ? max(key_begin[tok], 0) : 0, hi = key_end ? min(key_end[tok], total) : pos + 1;
  if (!valid || pos < 0 || hi <= lo) lo = 0x7fffffff, hi = 0;
  const bool none = hi == 0;
  // over the wavefront's rows: first begin, last begin, first end, last end
  const int w_lo = -lanes_max(0x7fffffff - lo) + 0x7fffffff, w_hi = lanes_max(hi), w_lo_last = lanes_max(none ? 0 : lo), w_hi_first = 0x7fffffff - lanes_max(none ? 0 : 0x7fffffff - hi);
  const bool given = key_begin || key_end;
  if (lane == 0) s_lo[wave] = w_lo, s_hi[wave] = w_hi;
  if (given) {
    // (a row without keys stands in for the nearest one of its wavefront that has some: those around it are neighbours then)
    const uint32_t some = (uint32_t)__ballot(!none), before = some & (0xffffffffu >> (31 - col));
    const int as = some ? before ? 31 - __builtin_clz(before) : __builtin_ctz(some) : col, as_lo = __shfl(lo, as), as_hi = __shfl(hi, as);
    if (half == 0) s_row_lo[wave * 32 + col] = as_lo, s_row_hi[wave * 32 + col] = as_hi;
  }
  if (tid < 2) s_bad[tid] = 0;
  __syncthreads();
  int t_lo = s_lo[0], t_hi = s_hi[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) t_lo = min(t_lo, s_lo[w]), t_hi = max(t_hi, s_hi[w]);
  t_lo = __builtin_amdgcn_readfirstlane(t_lo), t_hi = __builtin_amdgcn_readfirstlane(t_hi);
  // (without given ranges a row sees what the rows in front of it see)
  bool gaps = false;
  if (given) {
    const int n = min(rows - row0, W::kRows);
    bool apart = false;
#pragma unroll
    for (int i = 0; i < W::kRows; i += 64)
      if (const int r = i + lane; r + 1 < n) apart |= ranges_apart(s_row_lo[r], s_row_hi[r], s_row_lo[r + 1], s_row_hi[r + 1]);
    gaps = __any(apart);
  }
  uint16_t* const out_row = out + ((size_t)tok * Hq + head) * D;
  float* const lse_row = lse ? lse + (size_t)tok * Hq + head : nullptr;
  const int j_first = t_hi > 0 ? t_lo / kKeys : 0, j_end = t_hi > 0 ? (t_hi - 1) / kKeys + 1 : 0;
  const int splits = gridDim.y;
  const int j0 = __builtin_amdgcn_readfirstlane(j_first + (int)((long long)(j_end - j_first) * blockIdx.y / splits));
  const int j1 = __builtin_amdgcn_readfirstlane(j_first + (int)((long long)(j_end - j_first) * (blockIdx.y + 1) / splits));
  const int wj0 = __builtin_amdgcn_readfirstlane(w_hi > 0 ? w_lo / kKeys : 0), wj1 = __builtin_amdgcn_readfirstlane(w_hi > 0 ? (w_hi - 1) / kKeys + 1 : 0);

  bf16x8 qf[2 * NC];
  const uint16_t* const q_row = q + (size_t)tok * q_row_stride + (size_t)head * D;
#pragma unroll
  for (int t = 0; t < 2 * NC; ++t) {
    const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
    qf[t] = valid && 16 * t + 8 * half < D ? *reinterpret_cast<const bf16x8*>(q_row + 16 * t + 8 * half) : zero;
  }
  const float slope = (kForm == kBiased || kForm == kFarCapped) && form.slopes ? form.slopes[head] * kLog2e : 0.f;

  // ---- staging: a step's 16-byte pieces to registers, and from there to LDS as bf16
  const int blk_bytes = kBlockSize * D * C::kBytes;
  const uint32_t blk_stride = (uint32_t)Hkv * (uint32_t)blk_bytes;
  [[maybe_unused]] const uint32_t scale_stride = (uint32_t)Hkv * kScaleBytes;
  const char *const k_head = k_cache + (size_t)g * blk_bytes, *const v_head = v_cache + (size_t)g * blk_bytes;
  const int32_t* const table = block_table + (size_t)seq.b * bt_stride;
  const int blk_lo = t_lo >> 4, blk_hi = (t_hi - 1) >> 4;
  auto seen_in = [&](int j) { return seen_by_rows(s_row_lo, s_row_hi, W::kRows, j * kKeys); };
  u32x4 kr[W::kChunks], vr[W::kChunks];
  uint32_t k_scale = 127, v_scale[4] = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
  int id_k = 0, id_v = 0;
  const int v_block = wave & 3, v_part = wave >> 2;  // the block of V that the wavefront stages, and which of its runs of 64 places first
  uint64_t seen_asked = 0, seen_stored = 0;  // tiles with gaps: the keys that are seen, of the step whose blocks were named last and of the next one to be stored
  // (blocks without keys of the tile are not named: another of its blocks stands in, and is masked)
  auto load_ids = [&](int j, auto gapped) __attribute__((always_inline)) {
    constexpr bool kGaps = decltype(gapped)::value;
    if constexpr (kGaps) seen_asked = seen_in(j);
    id_k = table[entry_of_block(4 * j + (lane >> 4), blk_lo, blk_hi, kGaps, seen_asked)];
    id_v = table[entry_of_block(4 * j + v_block, blk_lo, blk_hi, kGaps, seen_asked)];
  };
  auto at_block = [](int id, uint32_t stride) { return (size_t)(uint32_t)id * stride; };
  auto load = [&]() __attribute__((always_inline)) {
    const char* const kp = k_head + at_block(id_k, blk_stride) + (lane & 15) * 16 + wave * 256;
    const char* const vp = v_head + at_block(id_v, blk_stride) + (v_part * 64 + lane) * 16;
#pragma unroll
    for (int i = 0; i < W::kChunks; ++i) {
      if (kFull || (kWaves * i + wave) * C::kUnit < D) kr[i] = *reinterpret_cast<const u32x4*>(kp + kWaves * 256 * i);  // unit kWaves i + wave
      if (kFull || (kWaves * 16 * i + v_part * 64 + lane) * 16 < blk_bytes) vr[i] = *reinterpret_cast<const u32x4*>(vp + kWaves * 256 * i);
    }
    if constexpr (W::kNarrow) {
      const uint8_t* const sc = scales + (size_t)g * kScaleBytes;
      k_scale = sc[at_block(id_k, scale_stride) + (lane & 15)];
      const u32x4 v = *reinterpret_cast<const u32x4*>(sc + at_block(id_v, scale_stride) + kBlockSize);
#pragma unroll
      for (int i = 0; i < 4; ++i) v_scale[i] = v[i];
    }
  };
  // (j: the step that lies in the registers)
  auto store = [&](int j, auto gapped) __attribute__((always_inline)) {
    char* const kb = s_k[W::kBuffers == 2 ? j & 1 : 0] + lane * 16;
    char* const vb = s_v[W::kBuffers == 2 ? j & 1 : 0] + 2 * v_block * W::kOctet + (W::kNarrow ? v_part * 1024 + lane * 16 : v_part * 512 + (lane >> 1) * 16 + (lane & 1) * W::kOctet);
    const u32x4 zero = {0, 0, 0, 0};
    const float ks = scale_of_byte(k_scale);
#pragma unroll
    for (int i = 0; i < W::kChunks; ++i) {
      const int u = kWaves * i + wave;
      const bool there = kFull || u * C::kUnit < D;
      if constexpr (W::kNarrow) {
        u32x4 a = zero, b = zero;
        if (there) {
          a = __builtin_bit_cast(u32x4, codes_to_bf16x8<F>(kr[i][0], kr[i][1], ks));
          b = __builtin_bit_cast(u32x4, codes_to_bf16x8<F>(kr[i][2], kr[i][3], ks));
        }
        *reinterpret_cast<u32x4*>(kb + 2 * u * kKeys * 16) = a;
        *reinterpret_cast<u32x4*>(kb + (2 * u + 1) * kKeys * 16) = b;
      } else {
        *reinterpret_cast<u32x4*>(kb + u * kKeys * 16) = there ? kr[i] : zero;
      }
    }
    // V: slots behind the tile's last key (nobody sees them) may hold anything: zeros.  So are those in front of the first, and between others that none of its rows sees.
    const int key0 = j * kKeys + 16 * v_block;
    uint32_t slots = 0xffffu;
    if constexpr (decltype(gapped)::value) slots &= (uint32_t)(seen_stored >> (16 * v_block));
    else if (key0 < t_lo || key0 + 16 > t_hi) slots &= (uint32_t)keys_seen(t_lo, t_hi, key0);
    const bool edge = slots != 0xffffu;
    if constexpr (W::kNarrow) {
      uint32_t sw[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) sw[w] = (uint32_t)__builtin_amdgcn_readfirstlane((int)v_scale[w]);
      auto clear = [&](const uint32_t (&keep)[4]) {  // (the slots' codes, and scales that say nothing)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          sw[w] = (sw[w] & keep[w]) | (0x7f7f7f7fu & ~keep[w]);
#pragma unroll
          for (int i = 0; i < W::kChunks; ++i) vr[i][w] &= keep[w];
        }
      };
      if (edge) {
        uint32_t keep[4] = {0, 0, 0, 0};
#pragma unroll
        for (int slot = 0; slot < 16; ++slot) keep[slot >> 2] |= slots >> slot & 1 ? 0xffu << (8 * (slot & 3)) : 0u;
        clear(keep);
      }
      // (a byte of 255 is a zero byte of ~w)
      auto any_bad = [&]() {
        uint32_t bad = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) bad |= (~sw[w] - 0x01010101u) & sw[w] & 0x80808080u;
        return bad != 0;
      };
      if (any_bad()) {
        uint32_t keep[4] = {0, 0, 0, 0};
#pragma unroll
        for (int slot = 0; slot < 16; ++slot) keep[slot >> 2] |= ((sw[slot >> 2] >> (8 * (slot & 3))) & 255u) != kBadScale ? 0xffu << (8 * (slot & 3)) : 0u;
        clear(keep);
        if (lane == 0) s_bad[j & 1] = j + 1;
      }
      // two tokens to a word: the conversion of e4m3 has one scale for both, so it is done with either, and a half of each kept
      float f[16];
#pragma unroll
      for (int w = 0; w < 4; ++w) f[4 * w] = scale_of<0>(sw[w]), f[4 * w + 1] = scale_of<1>(sw[w]), f[4 * w + 2] = scale_of<2>(sw[w]), f[4 * w + 3] = scale_of<3>(sw[w]);
#pragma unroll
      for (int i = 0; i < W::kChunks; ++i) {
        u32x4 x[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t c = vr[i][w];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float lo_scale = f[4 * w + 2 * h], hi_scale = f[4 * w + 2 * h + 1];
            uint32_t to;
            if constexpr (F == kE4m3) to = __builtin_amdgcn_perm(two_codes(c, hi_scale, h), two_codes(c, lo_scale, h), 0x07060100u);
            else to = h ? pack_bf16x2(code_value<F, 2>(c) * lo_scale, code_value<F, 3>(c) * hi_scale) : pack_bf16x2(code_value<F, 0>(c) * lo_scale, code_value<F, 1>(c) * hi_scale);
            x[w >> 1][2 * (w & 1) + h] = to;
          }
        }
        if (kFull || kWaves * 16 * i + v_part * 64 + lane < D) {
          *reinterpret_cast<u32x4*>(vb + kWaves * 256 * i) = x[0];
          *reinterpret_cast<u32x4*>(vb + kWaves * 256 * i + W::kOctet) = x[1];
        }
      }
    } else {
      if (edge) {
        const int h8 = 8 * (lane & 1);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int slot = h8 + 2 * w;
          const uint32_t keep = (slots >> slot & 1 ? 0xffffu : 0u) | (slots >> (slot + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
          for (int i = 0; i < W::kChunks; ++i) vr[i][w] &= keep;
        }
      }
#pragma unroll
      for (int i = 0; i < W::kChunks; ++i)
        if (kFull || kWaves * 8 * i + v_part * 32 + (lane >> 1) < D) *reinterpret_cast<u32x4*>(vb + kWaves * 128 * i) = vr[i];
    }
  };

  f32x16 o[NC];
#pragma unroll
  for (int dt = 0; dt < NC; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float m = kLowest, l = 0.f, poison = 0.f;

  // A-operand row -> key inside 32 keys: bits 2 and 3 swapped
  const int krow = (col & 0x13) | ((col & 4) << 1) | ((col & 8) >> 1);
  const int a_k_off = (half * kKeys + krow) * 16, a_v_off = half * W::kOctet + col * 16;

  auto step = [&](int j, auto) {
    const char* const kb = s_k[W::kBuffers == 2 ? j & 1 : 0] + a_k_off;
    const char* const vb = s_v[W::kBuffers == 2 ? j & 1 : 0] + a_v_off;
    f32x16 s[2];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[sub][i] = 0.f;
#pragma unroll
    for (int t = 0; t < 2 * NC; ++t)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(kb + (2 * t * kKeys + 32 * sub) * 16);
        s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[t], s[sub], 0, 0, 0);
      }
    const int k0 = j * kKeys;
    // register i of half-tile sub is key k0 + 32 sub + 16 (i / 8) + 8 half + i % 8
    if constexpr (kForm == kCapped) {
      // (the factor and the summand go with the maximum's into the weights' exponent)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[sub][i] = near_cap(s[sub][i], form.cap);
    }
    if constexpr (kForm == kFarCapped) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[sub][i] = far_cap(s[sub][i], form.cap);
    }
    if constexpr (kForm == kBiased || kForm == kFarCapped) {
      const float at_first = slope * (float)(k0 + 8 * half - pos);  // (the further keys' bias is slope times a literal)
      const float by = form.by, start = at_first + form.start;
      if (kForm == kBiased && form.cap.kind == kNear) {  // (one branch: as a choice per score it took as long as the products)
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[sub][i] = near_cap(s[sub][i], form.cap);
      }
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[sub][i] = __builtin_fmaf(slope, (float)(32 * sub + 16 * (i >> 3) + (i & 7)), __builtin_fmaf(s[sub][i], by, start));
    }
    if (k0 < w_lo_last || k0 + kKeys > w_hi_first) {
      asm volatile("" ::: "memory");  // (a branch, and no selects in every step)
      const unsigned from = (unsigned)(k0 + 8 * half - lo), keys = (unsigned)max(hi - lo, 0);
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * sub + 16 * (i >> 3) + (i & 7);
          if (from + at >= keys) s[sub][i] = -INFINITY;
        }
    }
    // the exponents of the weights: c s + shift
    const float c = kForm == kBiased || kForm == kFarCapped ? 1.f : form.by, at_zero = kForm == kCapped ? form.start : 0.f;
    float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) top = max3(top, s[0][i], s[0][i + 1]);
    top = max3(top, s[0][15], s[1][0]);
#pragma unroll
    for (int i = 1; i < 15; i += 2) top = max3(top, s[1][i], s[1][i + 1]);
    top = __builtin_fmaf(across_halves_max(fmaxf(top, s[1][15])), c, at_zero);
    if (__any(top > m)) {
      const float m_new = top > m ? top + kRoom : m, alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < NC; ++dt) o[dt] *= alpha;
      m = m_new;
    }
    const float shift = at_zero - m;
    u32x4 p[4];
    [[maybe_unused]] u32x4 second[4];
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 8 * (u & 1) + 2 * e;
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][i], c, shift)), b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][i + 1], c, shift));
        sums[0] += a;
        sums[1] += b;
        p[u][e] = first_parts<W::kTwo>(a, b);
        if constexpr (W::kTwo) second[u][e] = second_parts<true>(a, b, p[u][e]);
      }
    }
    l += sums[0] + sums[1];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int dt = 0; dt < NC; ++dt) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(vb + 2 * u * W::kOctet + 32 * dt * 16);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, p[u]), o[dt], 0, 0, 0);
        if constexpr (W::kTwo) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, second[u]), o[dt], 0, 0, 0);
      }
    if (W::kNarrow && s_bad[j & 1] == j + 1) {
      // a value's scale says NaN: rows that see it are NaN
      for (int at = max(lo, k0); at < min(hi, k0 + kKeys); ++at) {
        const int id = table[at >> 4];
        if (scales[((size_t)id * Hkv + g) * kScaleBytes + kBlockSize + (at & 15)] == kBadScale) poison = NAN;
      }
    }
  };

  // (a step is taken in where it is called, by word where there are two such places; where there is one the compiler does so by itself, after it has seen to the step alone: 4 x 4096 tokens, 8 heads on 1
  // of 256 over e4m3, 480 us by word and 445)
  auto walk = [&](auto gapped) __attribute__((always_inline)) {
    load_ids(j0, gapped);
    load();
    seen_stored = seen_asked;
    if (j0 + 1 < j1) load_ids(j0 + 1, gapped);
    store(j0, gapped);
    seen_stored = seen_asked;
    if (j0 + 1 < j1) {
      load();
      if (j0 + 2 < j1) load_ids(j0 + 2, gapped);
    }
    __syncthreads();
    for (int j = j0; j < j1; ++j) {
      if constexpr (W::kBuffers == 2) {
        // (of eight wavefronts that turn codes into operands, four do so first and four last, so that a SIMD's two are not at the same thing: 2170 and 2140 us of
        // two prompts of 8192 tokens; bf16 is only copied, and better all at once)
        const bool first = kWaves == 4 || !W::kNarrow || wave < 4;
        if (!first && j >= wj0 && j < wj1) [[clang::always_inline]] step(j, gapped);
        if (j + 1 < j1) {
          store(j + 1, gapped);
          seen_stored = seen_asked;
          if (j + 2 < j1) {
            load();
            if (j + 3 < j1) load_ids(j + 3, gapped);
          }
        }
        if (first && j >= wj0 && j < wj1) [[clang::always_inline]] step(j, gapped);
        __syncthreads();
      } else {
        if (j >= wj0 && j < wj1) step(j, gapped);
        __syncthreads();
        if (j + 1 < j1) {
          store(j + 1, gapped);
          seen_stored = seen_asked;
          if (j + 2 < j1) {
            load();
            if (j + 3 < j1) load_ids(j + 3, gapped);
          }
        }
        __syncthreads();
      }
    }
  };
  if (j0 < j1) {
    if constexpr (!kFull && !W::kNarrow) {
      // channels behind the head vector: no step writes them, and what is not finite there would have every row taken again
      for (int u = tid; u < W::kBuffers * 8 * (W::kD - D); u += W::kThreads) {
        const int at = u / (W::kD - D), d = D + u - at * (W::kD - D);
        *reinterpret_cast<u32x4*>(&s_v[0][0] + at / 8 * W::kVBytes + at % 8 * W::kOctet + d * 16) = u32x4{0, 0, 0, 0};
      }
    }
    // (two loops, so that the one of all other tiles has nothing to look for: in one, 2048 tokens of documents took 134 us instead of 128)
    if (gaps) walk(std::true_type());
    else walk(std::false_type());
  }
  l = across_halves_sum(l);
  if constexpr (W::kNarrow) {
#pragma unroll
    for (int dt = 0; dt < NC; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] += poison;
  }

  if (splits > 1) {
    // ---- parts of the steps: the states, in the lanes' own order; the last workgroup adds them up
    constexpr int kStateFloats = W::kRows * (32 * NC + 2);
    const size_t item = blockIdx.x;
    const __amdgpu_buffer_rsrc_t mine = __builtin_amdgcn_make_buffer_rsrc(states + (item * splits + blockIdx.y) * kStateFloats, 0, kStateFloats * 4, kRsrc);
    const int at = (wave * NC * 1024 + lane * 4) * 4, at_ml = (W::kRows * 32 * NC + 2 * (wave * 32 + col)) * 4;
#pragma unroll
    for (int dt = 0; dt < NC; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 v = {o[dt][4 * r], o[dt][4 * r + 1], o[dt][4 * r + 2], o[dt][4 * r + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), mine, at + (dt * 4 + r) * 1024, 0, kAgent);
      }
    if (half == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, mine, at_ml, 0, kAgent);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_order = (int)atomicInc(counters + item, (unsigned)splits - 1);
    __syncthreads();
    if (s_order != splits - 1) return;
    float M = kLowest;
    for (int k = 0; k < splits; ++k) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(states + (item * splits + k) * kStateFloats, 0, kStateFloats * 4, kRsrc);
      M = fmaxf(M, __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, at_ml, 0, kAgent)));
    }
    m = M;
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < NC; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    for (int k = 0; k < splits; ++k) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(states + (item * splits + k) * kStateFloats, 0, kStateFloats * 4, kRsrc);
      const u32x2 ml = __builtin_amdgcn_raw_buffer_load_b64(r, at_ml, 0, kAgent);
      const float w = __builtin_amdgcn_exp2f(__uint_as_float(ml[0]) - M);
      l += __uint_as_float(ml[1]) * w;
#pragma unroll
      for (int dt = 0; dt < NC; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + (dt * 4 + e) * 1024, 0, kAgent));
#pragma unroll
          for (int x = 0; x < 4; ++x) o[dt][4 * e + x] += v[x] * w;
        }
    }
  }

  // ---- results
  bool again = false;
  if constexpr (!W::kNarrow) {
    float odd = 0.f;  // NaN, if any result is not finite
#pragma unroll
    for (int dt = 0; dt < NC; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(o[dt][i], 0.f, odd);
    again = !none && across_halves_sum(odd) != 0.f && l < INFINITY;
    for (uint32_t left = (uint32_t)__ballot(again && half == 0); left; left &= left - 1) {
      const int r = __builtin_ctz(left);
      const int r_tok = __builtin_amdgcn_readlane(tok, r), r_head = __builtin_amdgcn_readlane(head, r), r_lo = __builtin_amdgcn_readlane(lo, r), r_hi = __builtin_amdgcn_readlane(hi, r);
      // (if nothing that the row does not see was the cause, the result stands)
      const int n = gaps ? W::kRows : 0;
      const bool unseen = not_finite_in(v_head, blk_stride, table, max(t_lo, wj0 * kKeys), r_lo, D, s_row_lo, s_row_hi, n) ||
                          not_finite_in(v_head, blk_stride, table, r_hi, min(t_hi, wj1 * kKeys), D, s_row_lo, s_row_hi, n);
      if (!unseen) {
        if (col == r) again = false;
        continue;
      }
      row_again<NC, kForm>(q + (size_t)r_tok * q_row_stride + (size_t)r_head * D, k_head, v_head, blk_stride, table, r_lo, r_hi, __builtin_amdgcn_readlane(pos, r),
                           __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(slope), r)), form, D, out + ((size_t)r_tok * Hq + r_head) * D);
    }
  }
  // Registers 4 i .. 4 i + 3 of o[dt] hold channels 32 dt + 8 i + 4 half + (0 .. 3).  The two lanes of a row exchange halves, so that each stores 16 bytes.
  const float inv = none ? 0.f : 1.f / l;
  auto pack = [&](float a, float b) { return none ? 0u : pack_bf16x2(a * inv, b * inv); };
#pragma unroll
  for (int dt = 0; dt < NC; ++dt)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const auto a = __builtin_amdgcn_permlane32_swap(pack(o[dt][8 * r], o[dt][8 * r + 1]), pack(o[dt][8 * r + 4], o[dt][8 * r + 5]), false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(pack(o[dt][8 * r + 2], o[dt][8 * r + 3]), pack(o[dt][8 * r + 6], o[dt][8 * r + 7]), false, false);
      const int d = 32 * dt + 16 * r + 8 * half;
      if (valid && !again && d < D) *reinterpret_cast<u32x4*>(out_row + d) = u32x4{a[0], b[0], a[1], b[1]};
    }
  if (lse_row && valid && half == 0) *lse_row = none ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int F, int NC, int kWaves>
void launch_waves(const ScoredArgs& a, int32_t splits, hipStream_t s) {
  const int G = a.Hq / a.Hkv, units = (int)prefill_scored_tiles(32 * kWaves, a.B, a.T, G);
  const Cap cap = make_cap(a.softcap, a.scale_log2e);
  const Form form = {cap, cap.kind == kNear ? 2.f * cap.log2e : cap.kind == kFar ? 1.f : a.scale_log2e, cap.kind == kNear ? cap.log2e : 0.f, a.slopes};
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)units * a.Hkv, (unsigned)splits), dim3(64 * kWaves), 0, s, (const uint16_t*)a.q, a.q_row_stride, (const char*)a.k_cache,
                       (const char*)a.v_cache, a.scales, a.cu_q, a.ctx_before, a.block_table, a.bt_stride, a.key_begin, a.key_end, (uint16_t*)a.out, a.lse, a.states,
                       a.counters, a.B, a.Hq, a.Hkv, G, make_divisor(G), make_divisor(a.Hkv), a.D, units, form);
  };
  const bool full = a.D == 32 * NC;
  auto with_form = [&](auto kind) {
    constexpr int kForm = decltype(kind)::value;
    full ? go(&prefill_scored_kernel<F, NC, kForm, true, kWaves>) : go(&prefill_scored_kernel<F, NC, kForm, false, kWaves>);
  };
  if (cap.kind == kFar) with_form(std::integral_constant<int, kFarCapped>());
  else if (a.slopes) with_form(std::integral_constant<int, kBiased>());
  else if (cap.kind == kNear) with_form(std::integral_constant<int, kCapped>());
  else with_form(std::integral_constant<int, kPlain>());
}

template <int F, int NC>
void launch_formed(const ScoredArgs& a, int32_t rows, int32_t splits, hipStream_t s) {
  if constexpr (NC == 4) {
    if (rows == kMostTileRows) return launch_waves<F, NC, 8>(a, splits, s);
  }
  launch_waves<F, NC, 4>(a, splits, s);
}

template <int F>
void launch_format(const ScoredArgs& a, int32_t rows, int32_t splits, hipStream_t s) {
  switch (scored_chunks(a.D)) {
    case 2: return launch_formed<F, 2>(a, rows, splits, s);
    case 4: return launch_formed<F, 4>(a, rows, splits, s);
    default: return launch_formed<F, 8>(a, rows, splits, s);
  }
}

}  // namespace

hipError_t launch_prefill_scored(const ScoredArgs& a, int32_t rows, int32_t splits, hipStream_t s) {
  switch (a.format) {
    case kInt8: launch_format<kInt8>(a, rows, splits, s); break;
    case kE4m3: launch_format<kE4m3>(a, rows, splits, s); break;
    default: launch_format<kNative>(a, rows, splits, s); break;
  }
  return hipGetLastError();
}

}  // namespace eco
