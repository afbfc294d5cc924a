// Block selection: every (token, K/V head) scores the summaries of its sequence's blocks and keeps the best.
//
// score(j) = max_h 2^(eq_h + e_j) sum_d max(q8 top_d, q8 low_d) is a product of whole numbers: max(q8 top, q8 low) =
// max(q8, 0) top + min(q8, 0) low, so with [max(q8, 0) | min(q8, 0)] as a row of 2 Dp and a block's record [top | low] as a
// column it is v_mfma_i32_16x16x64_i8, exact in 32 bits; scaled by a power of two it is exact in fp32 too.  Hence no
// order of sums, number of tokens or split of the blocks changes which blocks are chosen.
//
// Two launches, with the scores between them in the workspace, as unsigned numbers that are ordered as the scores are:
//   score_kernel   a wavefront has the rows (token, head of the group) of up to NA tiles of 16 as operands in registers and walks tiles of 16 blocks:
//                  16 bytes a lane and step, straight into operand layout.  The rows of a token are padded to a power of two with
//                  copies of its last head, so that the maximum over the heads is within a lane's four results and over
//                  at most two exchanges.  One token: bound by reading the records; prompts: by the products.
//   choose_kernel  a workgroup per (token, K/V head): a histogram of 2048 bins between the smallest and the largest
//                  number finds the bin that holds the last one to be chosen, then the same within that bin, until it is a
//                  single number or all of it is chosen; one prefix sum then writes the indices in their order.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "sparse.h"
#include "summary.h"

namespace eco {

namespace {

constexpr int kScoreThreads = 256, kScoreWaves = 4;
typedef int i32x4 __attribute__((ext_vector_type(4)));

// The tokens of a call: which sequence a token belongs to and where it stands.
struct Tokens {
  const int32_t *cu_q, *ctx_before;  // cu_q NULL: token b of sequence b
  int B, T;
};

// 16 elements of a query row from d on, as floats; zeros from D on.
template <typename E>
__device__ __forceinline__ void load16(const E* __restrict__ row, int d, int D, float (&x)[16]) {
  constexpr int X = Elem<E>::X;
#pragma unroll
  for (int u = 0; u < 16 / X; ++u) {
    u32x4 raw = {0u, 0u, 0u, 0u};
    if (d + u * X < D) raw = *reinterpret_cast<const u32x4*>(row + d + u * X);
#pragma unroll
    for (int e = 0; e < X; ++e)
      x[u * X + e] = sizeof(E) == 2 ? __uint_as_float(e & 1 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16) : __uint_as_float(raw[e % 4]);
  }
}

// Unsigned numbers in the order of the floats (no NaN; -0 counts as 0).  0 and 0xffffffff are no float's.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// NF: steps of 64 (record bytes / 64); NA: row tiles of a wavefront.  Grid: K/V heads, runs of tiles_per_wave * 4 block tiles, token groups from `unit0` on;
// a group is up to `group` tokens of one sequence, numbered from cu_q[b] / group + b.  Tokens outside [t0, t1) are another launch's.
template <typename E, int NF, int NA>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(const E* __restrict__ q, int q_row_stride, const int8_t* __restrict__ codes,
                                                               const int8_t* __restrict__ exponents, Tokens tk, const int32_t* __restrict__ block_table,
                                                               int bt_stride, uint32_t* __restrict__ scores, int64_t row_words, int G, int log_rows, int Hkv, int D,
                                                               int group, int unit0, int t0, int t1, int tiles_per_wave) {
  const int g = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
  // the group's tokens: first .. first + n - 1 of sequence b, the first at position p0
  int b, first, n, p0;
  if (tk.cu_q) {
    const int unit = unit0 + blockIdx.z;
    auto first_unit = [&](int cu, int s) { return (long long)(cu / group) + s; };
    const SeqOf seq = find_sequence(tk.cu_q, tk.ctx_before, tk.B, unit, first_unit);
    const int i0 = (int)(unit - first_unit(seq.tok0, seq.b)) * group;
    b = seq.b;
    first = max(seq.tok0 + i0, t0);
    n = min(min(seq.tok0 + i0 + group, seq.tok0 + seq.S), t1) - first;
    p0 = seq.cb + first - seq.tok0;
  } else {
    b = first = unit0 + blockIdx.z;
    n = first < t1 ? 1 : 0;
    p0 = n ? tk.ctx_before[b] : -1;
  }
  if (n <= 0 || p0 + n - 1 < 0) return;
  // the blocks that the group's last token scores: all in front of its own, which are full
  const int scored = (int)min((int64_t)((p0 + n - 1) >> 4), row_words);
  const int tile0 = (blockIdx.y * kScoreWaves + wave) * tiles_per_wave;
  if (tile0 * 16 >= scored) return;

  // operands of the rows: row r of tile a is head min(r % rows, G - 1) of token a * (16 / rows) + r / rows
  const int rows = 1 << log_rows, per_tile = 16 >> log_rows, Dp = NF * 32;
  i32x4 af[NA][NF];
  int eq[NA][4];
#pragma unroll
  for (int a = 0; a < NA; ++a) {
    const int tok = min(a * per_tile + (col >> log_rows), n - 1);
    const E* const row = q + (size_t)(first + tok) * q_row_stride + (size_t)(g * G + min(col & (rows - 1), G - 1)) * D;
    float size = 0.f, odd = 0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int k = f * 64 + quad * 16;
      float x[16];
      load16(row, k < Dp ? k : k - Dp, D, x);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        size = fmaxf(size, fabsf(x[i]));
        odd = __builtin_fmaf(x[i], 0.f, odd);
      }
    }
    size = fmaxf(size, __shfl_xor(size, 16));
    size = fmaxf(size, __shfl_xor(size, 32));
    odd += __shfl_xor(odd, 16);
    odd += __shfl_xor(odd, 32);
    const bool fine = odd == odd;
    const int e = fine ? code_exponent(size) : 0;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int k = f * 64 + quad * 16;
      float x[16];
      load16(row, k < Dp ? k : k - Dp, D, x);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t packed = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = fine ? (int)rintf(ldexpf(x[w * 4 + i], -e)) : 0;
          packed |= ((uint32_t)(k < Dp ? max(c, 0) : min(c, 0)) & 0xffu) << (8 * i);
        }
        af[a][f][w] = (int)packed;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) eq[a][i] = __shfl(e, quad * 4 + i);
  }

  const int32_t* const table = block_table + (size_t)b * bt_stride;
  const int tile1 = min(tile0 + tiles_per_wave, (scored + 15) >> 4);
  auto block_at = [&](int tile) { return (int64_t)table[min(tile * 16 + col, scored - 1)]; };
  uint32_t* const out = scores + ((int64_t)(first - t0) * Hkv + g) * row_words;
  auto load = [&](i32x4 (&bf)[NF], int& e, int64_t blk) {
    const int8_t* const rec = codes + ((size_t)blk * Hkv + g) * (2 * Dp) + quad * 16;
#pragma unroll
    for (int f = 0; f < NF; ++f) bf[f] = *reinterpret_cast<const i32x4*>(rec + f * 64);
    e = exponents[(size_t)blk * Hkv + g];
  };
  i32x4 bf[NF], next[NF];
  int e, e_next = 0;
  load(bf, e, block_at(tile0));
  int64_t blk = block_at(min(tile0 + 1, tile1 - 1));
  for (int tile = tile0; tile < tile1; ++tile) {
    load(next, e_next, blk);
    blk = block_at(min(tile + 2, tile1 - 1));
#pragma unroll
    for (int a = 0; a < NA; ++a) {
      if (a * per_tile >= n) break;
      i32x4 c = {0, 0, 0, 0};
#pragma unroll
      for (int f = 0; f < NF; ++f) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(af[a][f], bf[f], c, 0, 0, 0);
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = ldexpf((float)c[i], eq[a][i] + e);
      // the maximum over a token's rows; it is then in v[0] (and, for one or two rows a token, v[2] or all four)
      if (log_rows >= 1) v[0] = fmaxf(v[0], v[1]), v[2] = fmaxf(v[2], v[3]);
      if (log_rows >= 2) v[0] = fmaxf(v[0], v[2]);
      if (log_rows >= 3) v[0] = fmaxf(v[0], __shfl_xor(v[0], 16));
      if (log_rows >= 4) v[0] = fmaxf(v[0], __shfl_xor(v[0], 32));
      const int step = log_rows < 2 ? rows : 4;  // v[0], v[step], .. are tokens of their own
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i & (step - 1)) continue;
        const int row = quad * 4 + i, tok = a * per_tile + (row >> log_rows);
        if ((row & (rows - 1)) == 0 && tok < n) out[(int64_t)tok * Hkv * row_words + tile * 16 + col] = ordered(e == kNotFinite ? INFINITY : v[i]);
      }
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) bf[f] = next[f];
    e = e_next;
  }
}

constexpr int kBins = 2048, kPer = 8;  // bins of a histogram; numbers of a thread at a time

// Inclusive sums over the workgroup of two counts; `all`: their totals.
template <int THREADS>
__device__ __forceinline__ int2 sum_over_threads(int2 x, int2* s_wave, int2& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x.x = lanes_prefix_sum(x.x);
  x.y = lanes_prefix_sum(x.y);
  __syncthreads();
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  all = int2{0, 0};
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const int2 y = s_wave[w];
    if (w < wave) x.x += y.x, x.y += y.y;
    all.x += y.x, all.y += y.y;
  }
  return x;
}

// Grid: K/V heads, tokens t0 .. t1 - 1.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void choose_kernel(const uint32_t* __restrict__ scores, int64_t row_words, Tokens tk, int32_t* __restrict__ blocks, int K,
                                                         int keep_first, int keep_last, int Hkv, int t0) {
  __shared__ int s_hist[kBins];
  __shared__ int2 s_wave[THREADS / 64];
  __shared__ uint32_t s_low[THREADS / 64], s_high[THREADS / 64];
  __shared__ int s_bin, s_above;
  const int g = blockIdx.x, t = t0 + blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int p;
  if (tk.cu_q) {
    const SeqOf seq = find_sequence(tk.cu_q, tk.ctx_before, tk.B, t, [](int cu, int) { return (long long)cu; });
    if (t - seq.tok0 >= seq.S) return;  // (behind the last sequence)
    p = seq.cb + t - seq.tok0;
  } else {
    p = tk.ctx_before[t];
  }
  const int n = p < 0 ? 0 : (int)min((int64_t)(p >> 4) + 1, row_words);
  int32_t* const out = blocks + ((int64_t)t * Hkv + g) * K;
  if (n <= K) {
    for (int i = tid; i < K; i += THREADS) out[i] = i < n ? i : -1;
    return;
  }
  const uint32_t* const row = scores + ((int64_t)(t - t0) * Hkv + g) * row_words;
  constexpr int kSpan = THREADS * kPer;
  const int c0 = keep_first, c1 = n - keep_last;  // the blocks that compete
  int need = K - keep_first - keep_last;
  uint32_t key[kPer];
  // numbers base + 8 tid .. + 7: 0 behind the last block, the largest for what is kept anyway
  auto load = [&](int base) {
    const int j0 = base + tid * kPer;
#pragma unroll
    for (int w = 0; w < kPer / 4; ++w) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (j0 + 4 * w < c1) x = *reinterpret_cast<const u32x4*>(row + j0 + 4 * w);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = j0 + 4 * w + i;
        key[4 * w + i] = j >= n ? 0u : j < c0 || j >= c1 ? ~0u : x[i];
      }
    }
  };
  const bool once = n <= kSpan;  // all of them in registers
  load(0);
  // the smallest number that is chosen and how many equal to it are: `at` and `need`
  uint32_t at = ~0u;
  bool whole = true;  // all numbers from `at` on are chosen
  if (need > 0) {
    uint32_t low = ~0u, high = 0u;
    for (int base = 0; base < n; base += kSpan) {
      if (!once) load(base);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (key[i] != 0u && key[i] != ~0u) low = min(low, key[i]), high = max(high, key[i]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) low = min(low, (uint32_t)__shfl_xor((int)low, o)), high = max(high, (uint32_t)__shfl_xor((int)high, o));
    if (lane == 0) s_low[wave] = low, s_high[wave] = high;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) low = min(low, s_low[w]), high = max(high, s_high[w]);
    uint32_t span = high - low;  // numbers low .. low + span
    for (;;) {
      const int shift = max(0, 32 - __clz((int)(span | 1u)) - 11);
      __syncthreads();
      for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
      __syncthreads();
      for (int base = 0; base < n; base += kSpan) {
        if (!once) load(base);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (key[i] != 0u && key[i] != ~0u && key[i] >= low && key[i] - low <= span) atomicAdd(&s_hist[(key[i] - low) >> shift], 1);
      }
      __syncthreads();
      // from the last bin down: the one in which the count reaches `need`
      constexpr int kBinsPer = kBins / THREADS;
      int mine = 0, bins[kBinsPer];
#pragma unroll
      for (int i = 0; i < kBinsPer; ++i) {
        bins[i] = s_hist[kBins - 1 - (tid * kBinsPer + i)];
        mine += bins[i];
      }
      int2 all;
      int above = sum_over_threads<THREADS>(int2{mine, 0}, s_wave, all).x - mine;
#pragma unroll
      for (int i = 0; i < kBinsPer; ++i) {
        if (above < need && above + bins[i] >= need) s_bin = kBins - 1 - (tid * kBinsPer + i), s_above = above;
        above += bins[i];
      }
      __syncthreads();
      const int bin = s_bin;
      need -= s_above;
      at = low + ((uint32_t)bin << shift);
      whole = need == s_hist[bin];
      if (whole || shift == 0) break;
      low = at;
      span = (1u << shift) - 1u;
    }
  }
  // indices in their order: all numbers above `at`, and of those equal to it the first `need`
  int done = 0, equal = 0;
  for (int base = 0; base < n; base += kSpan) {
    if (!once) load(base);
    int2 mine = {0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool sure = key[i] != 0u && (whole ? key[i] >= at : key[i] > at);
      mine.x += sure ? 1 : 0;
      mine.y += !whole && key[i] == at ? 1 : 0;
    }
    int2 all;
    const int2 upto = sum_over_threads<THREADS>(mine, s_wave, all);
    int sure_before = done + upto.x - mine.x, equal_before = equal + upto.y - mine.y;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool sure = key[i] != 0u && (whole ? key[i] >= at : key[i] > at), same = !whole && key[i] == at;
      if (sure || (same && equal_before < need)) out[sure_before + min(equal_before, need)] = base + tid * kPer + i;
      sure_before += sure ? 1 : 0;
      equal_before += same ? 1 : 0;
    }
    done += all.x;
    equal += all.y;
  }
}

template <typename E, int NF, int NA>
void launch_scores(const SelectArgs& a, const Tokens& tk, const int8_t* codes, const int8_t* exponents, int64_t row_words, int log_rows, int group, int t0, int t1,
                   hipStream_t s) {
  const int G = a.Hq / a.Hkv, tiles = (int)(row_words / 16);
  // tokens t of sequence b are in unit t / group + b or the one in front of it
  const int unit0 = a.cu_q ? std::max(0, t0 / group - 1) : t0, units = a.cu_q ? t1 / group + a.B + 1 - unit0 : t1 - t0;
  // as many wavefronts as the device takes at once, then more tiles to one
  const int64_t waves = (int64_t)units * a.Hkv * tiles, room = (int64_t)a.num_cu * 16;
  const int per_wave = (int)std::min<int64_t>(std::max<int64_t>(1, waves / room), 16), runs = (tiles + kScoreWaves * per_wave - 1) / (kScoreWaves * per_wave);
  hipLaunchKernelGGL((score_kernel<E, NF, NA>), dim3((unsigned)a.Hkv, (unsigned)runs, (unsigned)units), dim3(kScoreThreads), 0, s, (const E*)a.q, a.q_row_stride,
                     codes, exponents, tk, a.block_table, a.bt_stride, a.scores, row_words, G, log_rows, a.Hkv, a.D, group, unit0, t0, t1, per_wave);
}

template <typename E>
void launch_typed(const SelectArgs& a, const Tokens& tk, const int8_t* codes, const int8_t* exponents, int64_t row_words, int t0, int t1, hipStream_t s) {
  const int G = a.Hq / a.Hkv;
  int log_rows = 0;
  while ((1 << log_rows) < G) ++log_rows;
  const bool prompts = a.cu_q && a.T > 2 * a.B;
  auto steps = [&](auto nf) {
    constexpr int NF = decltype(nf)::value, NA = NF <= 4 ? 4 : 2;
    if (prompts) launch_scores<E, NF, NA>(a, tk, codes, exponents, row_words, log_rows, NA * (16 >> log_rows), t0, t1, s);
    else launch_scores<E, NF, 1>(a, tk, codes, exponents, row_words, log_rows, a.cu_q ? 16 >> log_rows : 1, t0, t1, s);
  };
  switch (summary_channels(a.D) / 32) {
    case 1: return steps(std::integral_constant<int, 1>());
    case 2: return steps(std::integral_constant<int, 2>());
    case 3: return steps(std::integral_constant<int, 3>());
    case 4: return steps(std::integral_constant<int, 4>());
    case 5: return steps(std::integral_constant<int, 5>());
    case 6: return steps(std::integral_constant<int, 6>());
    case 7: return steps(std::integral_constant<int, 7>());
    default: return steps(std::integral_constant<int, 8>());
  }
}

}  // namespace

hipError_t launch_block_select(const ecoserve_layout& L, const SelectArgs& a, const void* summary, int32_t max_ctx_len, hipStream_t s) {
  const int8_t* const codes = (const int8_t*)summary;
  const int8_t* const exponents = codes + summary_code_bytes(L);
  const Tokens tk = {a.cu_q, a.ctx_before, a.B, a.T};
  const int64_t row_words = select_row_words(max_ctx_len);
  const int at_a_time = select_tokens_at_a_time(L.num_kv_heads, a.T, max_ctx_len);
  for (int t0 = 0; t0 < a.T; t0 += at_a_time) {
    const int t1 = std::min(a.T, t0 + at_a_time);
    // (no more blocks than are asked for, whatever the lengths: nothing is scored)
    if (row_words > a.num_selected) {
      if (L.dtype == ECOSERVE_BF16) launch_typed<uint16_t>(a, tk, codes, exponents, row_words, t0, t1, s);
      else launch_typed<float>(a, tk, codes, exponents, row_words, t0, t1, s);
    }
    const dim3 grid((unsigned)a.Hkv, (unsigned)(t1 - t0));
    if (row_words <= 256 * kPer)
      hipLaunchKernelGGL((choose_kernel<256>), grid, dim3(256), 0, s, a.scores, row_words, tk, a.blocks, a.num_selected, a.keep_first, a.keep_last, a.Hkv, t0);
    else
      hipLaunchKernelGGL((choose_kernel<1024>), grid, dim3(1024), 0, s, a.scores, row_words, tk, a.blocks, a.num_selected, a.keep_first, a.keep_last, a.Hkv, t0);
  }
  return hipGetLastError();
}

}  // namespace eco
