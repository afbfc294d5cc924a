// Block selection: every (token, K/V head) scores the summaries of its sequence's blocks and keeps the best.
//
// score(j) = max_h 2^(eq_h + e_j) sum_d max(q8 top_d, q8 low_d) is a product of whole numbers: max(q8 top, q8 low) =
// max(q8, 0) top + min(q8, 0) low, so with [max(q8, 0) | min(q8, 0)] as a row of 2 Dp and a block's record [top | low] as a
// column it is v_mfma_i32_16x16x64_i8, exact in 32 bits; scaled by a power of two it is exact in fp32 too (a sum of exponents
// outside -149 .. 106 takes it beyond fp32: it is infinite there, or rounded to subnormals).  Hence no
// order of sums, number of tokens or split of the blocks changes which blocks are chosen.
//
// The rows of a product are (token, head of the group), a token's padded to a power of two with copies of its last head, so that the
// maximum over the heads is within a lane's four results and over at most two exchanges; its columns are 16 blocks, 16 bytes a lane and step, straight into
// operand layout.
//   score_step_kernel    few tokens per sequence: a workgroup codes up to 16 rows into LDS and walks a run of block tiles.  Bound by reading the
//                        records, 256 bytes per head of each of a table's scattered blocks (32 sequences of 16384 to 131000 tokens, 8 heads of 128, 0.3 GB: 67 us,
//                        4.5 TB/s).
//   code_kernel, score_prompt_kernel   prompts: the rows are coded once, into the workspace; a wavefront has four tiles of them in registers.  Bound by the
//                        products and the instructions on their results (895 tokens, 64 heads on 8 of 128, about 1500 blocks: 33.3 us; either alone would take about 9).
//   choose               a wavefront or more per (token, K/V head), the scores in registers.  For steps over short contexts the workgroup that is
//                        done last with a row's scores does it in the same launch, otherwise choose_kernel.
// The scores go through the workspace.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "sparse.h"
#include "summary.h"

namespace eco {

namespace {

constexpr int kScoreThreads = 256, kScoreWaves = 4;
constexpr float kLargestQuery = 127.f * 0x1p100f;  // query heads beyond it are coded as zeros: a sum of products times 2^eq then stays in range
typedef int i32x4 __attribute__((ext_vector_type(4)));

// The tokens of a call: which sequence a token belongs to and where it stands.
struct Tokens {
  const int32_t *cu_q, *ctx_before;  // cu_q NULL: token b of sequence b
  int B, T;
};

// What a row is chosen into.
struct Chosen {
  int32_t* blocks;
  int K, keep_first, keep_last;
};

// The maximum over lanes 16 (32) apart: a's in the first of each two rows (halves) of lanes, b's in the second.
__device__ __forceinline__ float max_of_rows16(float a, float b) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float max_of_rows32(float a, float b) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
// The maximum over the 16 lanes of a row of lanes.
__device__ __forceinline__ float max_in_row(float v) {
  auto with = [&](auto ctrl) {
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  with(std::integral_constant<int, 0xB1>());   // quad_perm 1 0 3 2
  with(std::integral_constant<int, 0x4E>());   // quad_perm 2 3 0 1
  with(std::integral_constant<int, 0x141>());  // row_half_mirror
  with(std::integral_constant<int, 0x140>());  // row_mirror
  return v;
}

// A query head as whole numbers, by the 16 lanes of a row of lanes: `ask` has its 16-byte units on the way, `code` writes [max(q8, 0) | min(q8, 0)] to
// `to` and returns 2^eq.
template <typename E, int NF>
struct CodedRow {
  static constexpr int X = Elem<E>::X, kUnits = (NF * 32 / X + 15) / 16;
  u32x4 raw[kUnits];
  __device__ __forceinline__ void ask(const E* __restrict__ row, int D, int col) {
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int d = (col + 16 * k) * X;
      raw[k] = d < D ? *reinterpret_cast<const u32x4*>(row + d) : u32x4{0u, 0u, 0u, 0u};
    }
  }
  __device__ __forceinline__ float code(int8_t* to, int col) const {
    constexpr int Dp = NF * 32;
    float x[kUnits][X], size = 0.f;
    bool fine = true;
#pragma unroll
    for (int k = 0; k < kUnits; ++k)
#pragma unroll
      for (int i = 0; i < X; ++i) {
        x[k][i] = sizeof(E) == 2 ? __uint_as_float(i & 1 ? raw[k][i / 2] & 0xffff0000u : raw[k][i / 2] << 16) : __uint_as_float(raw[k][i % 4]);
        size = fmaxf(size, fabsf(x[k][i]));
        fine = fine && x[k][i] == x[k][i];
      }
    size = max_in_row(fine ? size : INFINITY);
    fine = size <= kLargestQuery;
    const int e = code_exponent(size);
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      uint32_t top[X / 4], low[X / 4];
#pragma unroll
      for (int w = 0; w < X / 4; ++w) {
        top[w] = low[w] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = fine ? (int)rintf(ldexpf(x[k][w * 4 + i], -e)) : 0;
          top[w] |= ((uint32_t)max(c, 0) & 0xffu) << (8 * i);
          low[w] |= ((uint32_t)min(c, 0) & 0xffu) << (8 * i);
        }
      }
      const int d = (col + 16 * k) * X;
      if (d >= Dp) continue;
      if constexpr (X == 8) {
        *reinterpret_cast<u32x2*>(to + d) = u32x2{top[0], top[1]};
        *reinterpret_cast<u32x2*>(to + Dp + d) = u32x2{low[0], low[1]};
      } else {
        *reinterpret_cast<uint32_t*>(to + d) = top[0];
        *reinterpret_cast<uint32_t*>(to + Dp + d) = low[0];
      }
    }
    return fine ? ldexpf(1.f, e) : 1.f;
  }
};

// The numbers of a row in order: the larger the score the larger the number.  (No NaN; -0 counts as 0; 0 is no score's number.)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Choosing the largest of a row's numbers: histograms, two that are used in turn, with a bin per lane for what is not counted, and what the wavefronts tell one
// another.
template <int WAVES, int BINS>
struct ChooseShared {
  alignas(16) int hist[2][BINS + 64];
  uint32_t low[WAVES], high[WAVES], left[64];
  int sures[WAVES], sames[WAVES], n_left;
};
template <int WAVES>
__device__ __forceinline__ void together() {
  if constexpr (WAVES > 1) {
    __syncthreads();
  } else {  // (a wavefront by itself: its LDS accesses take effect in their order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// K of the n blocks of a row, ascending, to `out`: all outside [c0, c1), and of those inside, whose scores are ask(j), the best; lower indices first
// among equal ones.  n > K.  Each wavefront has a run of indices, a lane every 64th: PER of them, in registers, or, PER 0, as many as it takes, asked for
// again each time.  A histogram between the smallest and the largest number finds the bin in which the last one to be chosen is.  Up to 64 numbers of
// that bin are then compared with one another, a lane each, bit by bit; of more, another histogram is made.  Every wavefront does all of that but the counting
// by itself: a barrier or two a round.  What bounds it is instructions, their fetching where a row is alone: hence no branch per number.
// (895 tokens, 8 K/V heads, about 1500 blocks, a wavefront a row, us: loads and counts under branches 36.1, loads at once 27.0, so 20.2.)
template <int WAVES, int PER, int BINS, typename Ask>
__device__ __forceinline__ void choose(Ask ask, int wave, int n, int c0, int c1, int K, int32_t* __restrict__ out, ChooseShared<WAVES, BINS>& s) {
  constexpr int THREADS = WAVES * 64, kMine = BINS / 64, kLog = BINS == 1024 ? 10 : 9, kAll = 2 * (BINS + 64);
  static_assert(BINS == 1 << kLog, "bins");
  const int lane = threadIdx.x & 63, tid = wave * 64 + lane;
  const int run = PER > 0 ? PER * 64 : (n + THREADS - 1) / THREADS * 64, j0 = wave * run + lane;
  // 0: no block; the largest: chosen whatever its score
  auto number = [&](float x, int j) { return j >= n ? 0u : j < c0 || j >= c1 ? ~0u : ordered(x); };
  uint32_t key[PER > 0 ? PER : 1];
  if constexpr (PER > 0) {
    float x[PER];  // (all asked for at once, the last one in place of those behind it)
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = ask(min(j0 + i * 64, c1 - 1));
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = number(x[i], j0 + i * 64);
  }
  auto each = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (i % 8 == 0 && wave * run + i * 64 >= n) break;
        f(key[i], j0 + i * 64);
      }
    } else {
      for (int j = j0; j - lane < min(n, (wave + 1) * run); j += 64) f(number(ask(min(j, c1 - 1)), j), j);
    }
  };
  int need = K - (n - (c1 - c0));
  uint32_t at = ~0u - 1u;  // all numbers above it are chosen, and `need` of those equal to it
  if (need > 0) {
    uint32_t low = ~0u, high = 0u;
    each([&](uint32_t k, int) {  // (0 becomes the largest for one, the largest 0 for the other)
      low = min(low, k - 1u);
      high = max(high, k + 1u);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) low = min(low, (uint32_t)__shfl_xor((int)low, o)), high = max(high, (uint32_t)__shfl_xor((int)high, o));
    for (int i = tid * 4; i < kAll; i += THREADS * 4) *reinterpret_cast<u32x4*>(&s.hist[0][0] + i) = u32x4{0u, 0u, 0u, 0u};
    if (tid == 0) s.n_left = 0;
    if (WAVES > 1 && lane == 0) s.low[wave] = low, s.high[wave] = high;
    together<WAVES>();
    if (WAVES > 1)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) low = min(low, s.low[w]), high = max(high, s.high[w]);
    ++low;
    uint32_t span = high - 1u - low;  // numbers low .. low + span
    for (int turn = 0;; turn ^= 1) {
      const int shift = max(0, 32 - kLog - __clz((int)(span | 1u)));
      each([&](uint32_t k, int) {
        const uint32_t d = k - low;
        atomicAdd(&s.hist[turn][d <= span ? d >> shift : BINS + lane], 1);
      });
      together<WAVES>();
      // from the last bin down, a lane kMine of them: the bin in which the count reaches `need`
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kMine; i += 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(&s.hist[turn][BINS - 4 - lane * kMine - i]);
        mine += (int)(x[0] + x[1]) + (int)(x[2] + x[3]);
      }
      const int upto = lanes_prefix_sum(mine);
      const int l = __builtin_ctzll(__ballot(upto >= need) | 1ull << 63);  // the lane that has it
      need -= __builtin_amdgcn_readlane(upto - mine, l);
      // (its bins, a lane each)
      const int one = lane < kMine ? s.hist[turn][BINS - 1 - l * kMine - min(lane, kMine - 1)] : 0, to = lanes_prefix_sum(one);
      const int b = __builtin_ctzll(__ballot(to >= need) | 1ull << 63), in_bin = __builtin_amdgcn_readlane(one, b);
      need -= __builtin_amdgcn_readlane(to - one, b);
      low += (uint32_t)(BINS - 1 - l * kMine - b) << shift;
      if (need == in_bin) {  // all of the bin
        at = low - 1;
        need = 0;
        break;
      }
      if (shift == 0) {
        at = low;
        break;
      }
      span = (1u << shift) - 1u;
      if (in_bin <= 64) {
        each([&](uint32_t k, int) {
          const bool in = k - low <= span;
          if (__any(in)) {
            if (in) s.left[atomicAdd(&s.n_left, 1) & 63] = k - low;
          }
        });
        together<WAVES>();
        const uint32_t d = lane < in_bin ? s.left[lane] : 0u;
        uint32_t found = 0;  // the largest number that at least `need` of them reach
        for (uint32_t bit = 1u << (shift - 1); bit; bit >>= 1)
          if (__popcll(__ballot(lane < in_bin && d >= (found | bit))) >= need) found |= bit;
        need -= __popcll(__ballot(lane < in_bin && d > found));
        at = low + found;
        if (need == __popcll(__ballot(lane < in_bin && d == found))) --at, need = 0;  // (all of them)
        break;
      }
      // the histogram of the round after the next
      together<WAVES>();
      for (int i = tid * 4; i < BINS; i += THREADS * 4) *reinterpret_cast<u32x4*>(&s.hist[turn][i]) = u32x4{0u, 0u, 0u, 0u};
    }
  }
  // how many each wavefront has, then where they go
  auto before = [&](unsigned long long m) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u)); };
  int sures = 0, sames = 0;
  if (WAVES > 1) {
    each([&](uint32_t k, int) {
      sures += __popcll(__ballot(k > at));
      sames += __popcll(__ballot(k == at));
    });
    if (lane == 0) s.sures[wave] = sures, s.sames[wave] = sames;
    together<WAVES>();
    sures = sames = 0;
    for (int w = 0; w < wave; ++w) sures += s.sures[w], sames += s.sames[w];
  }
  if (need == 0) {
    each([&](uint32_t k, int j) {
      const unsigned long long m = __ballot(k > at);
      if (k > at) out[min(sures + before(m), K - 1)] = j;
      sures += __popcll(m);
    });
  } else {
    each([&](uint32_t k, int j) {
      const unsigned long long m0 = __ballot(k > at), m1 = __ballot(k == at);
      const int nth_same = sames + before(m1);
      if (k > at || (k == at && nth_same < need)) out[min(sures + before(m0) + min(nth_same, need), K - 1)] = j;
      sures += __popcll(m0);
      sames += __popcll(m1);
    });
  }
}

// Scores of a row, from one workgroup to another within a launch and possibly between XCDs: past the caches that XCDs do not share.
constexpr int kRsrc = 0x00020000, kAgent = 16;
// Scores of n tokens for one K/V head, from the first one's row on (below 2 GiB: more than one token at a time have 192 MiB).
constexpr int kNowhere = 0x7fff0000;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t score_rows(float* out, int n, int Hkv, int64_t row_words) {
  return __builtin_amdgcn_make_buffer_rsrc(out, 0, (int)(((int64_t)(n - 1) * Hkv + 1) * row_words * 4), kRsrc);
}
// (no branch around a store: it would have everything waited for that is under way)
template <int AUX>
__device__ __forceinline__ void put_score(__amdgpu_buffer_rsrc_t to, int where, int tile, float v, int e) {
  const float score = e == kNotFinite ? INFINITY : ldexpf(v, e);
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(score), to, where, tile * 64, AUX);
}

// A tile of 16 records, from memory to LDS to operands.  A lane's operand is 16 bytes of "its" block, so loads straight into operand layout would have
// neighbouring lanes ask different lines, 64 requests an instruction (895 tokens: 62 us; steps over 32 long contexts: 64);
// so lanes ask for 64 bytes in a row per four, and LDS turns them over: 38 us and, bound by the records' places, 64 as before.  Unit s (16 bytes) of block c lies at unit s ^ mix(c) of its
// row, which has the 16 blocks' units of any step at different banks.
template <int NF>
struct Records {
  static constexpr int kUnits = 4 * NF, kBytes = 16 * kUnits * 16, kBits = NF % 4 == 0 ? 4 : NF % 2 == 0 ? 3 : 2;
  u32x4 raw[NF];
  int e;
  static __device__ __forceinline__ int mix(int c) { return c >> (4 - kBits); }
  // id: the block of lanes c, c + 16, ..
  __device__ __forceinline__ void ask(const int8_t* __restrict__ codes, const int8_t* __restrict__ exponents, int id, int g, int Hkv, int lane) {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int u = i * 64 + lane, c = u / kUnits, s = (u - c * kUnits) ^ mix(c);
      raw[i] = *reinterpret_cast<const u32x4*>(codes + ((size_t)__shfl(id, c) * Hkv + g) * (kUnits * 16) + s * 16);
    }
    e = exponents[(size_t)id * Hkv + g];
  }
  __device__ __forceinline__ void put(char* tile, int lane) const {
#pragma unroll
    for (int i = 0; i < NF; ++i) *reinterpret_cast<u32x4*>(tile + (i * 64 + lane) * 16) = raw[i];
  }
  static __device__ __forceinline__ void get(i32x4 (&bf)[NF], const char* tile, int col, int quad) {
#pragma unroll
    for (int f = 0; f < NF; ++f) bf[f] = *reinterpret_cast<const i32x4*>(tile + (col * kUnits + ((4 * f + quad) ^ mix(col))) * 16);
  }
};

// NF: steps of 64 (record bytes / 64).  Grid: K/V heads, 1 << log_heads of them a workgroup, runs of tiles_per_wave block tiles for each wavefront of a head,
// token groups from `unit0` on; a group is up to `group` tokens of one sequence, numbered from cu_q[b] / group + b.  Tokens outside [t0, t1) are another launch's.  PER > 0 (one token per sequence, rows of at most 256 PER blocks):
// the workgroup that is done last with a row chooses its blocks; counters [T][Hkv] are zero and stay so.
template <typename E, int NF, int PER>
__global__ __launch_bounds__(kScoreThreads) void score_step_kernel(const E* __restrict__ q, int q_row_stride, const int8_t* __restrict__ codes,
                                                                    const int8_t* __restrict__ exponents, Tokens tk, const int32_t* __restrict__ block_table,
                                                                    int bt_stride, float* __restrict__ scores, int64_t row_words, int G, int log_rows, int Hkv, int D,
                                                                    int group, int unit0, int t0, int t1, int tiles_per_wave, int log_heads, Chosen to,
                                                                    uint32_t* __restrict__ counters) {
  constexpr int Dp = NF * 32, kRow = 2 * Dp + 16;  // bytes of a coded row in LDS, 16 more than it has: rows begin at different banks
  constexpr bool kChoose = PER > 0;
  struct Coded {
    float scale[16];
    alignas(16) int8_t row[16 * kRow];
  };
  // the coded rows of the heads, then each wavefront's tile
  constexpr int kHeads = kChoose ? 1 : kScoreWaves, kTiles = kScoreWaves * Records<NF>::kBytes, kCoded = kHeads * (int)sizeof(Coded);
  __shared__ __attribute__((aligned(16))) char s_any[kTiles > kCoded ? kTiles : kCoded];
  Coded* const coded = reinterpret_cast<Coded*>(s_any);
  __shared__ ChooseShared<kScoreWaves, kChoose ? 1024 : 512> s_choose;
  __shared__ int s_order;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
  // this wavefront: a head of the workgroup's, and every `phases`th tile
  const int heads = kChoose ? 1 : 1 << log_heads, phases = kChoose ? kScoreWaves : kScoreWaves >> log_heads;
  const int g0 = blockIdx.x * heads, here = kChoose ? 0 : wave & (heads - 1), phase = kChoose ? wave : wave >> log_heads, g = g0 + here;
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
    if (n <= 0 || p0 + n - 1 < 0) return;
  } else {
    b = first = unit0 + blockIdx.z;
    n = 1;
    p0 = tk.ctx_before[b];
  }
  // a row to each 16 lanes, asked for before anything is known of the lengths
  const int r = wave * 4 + quad, r_tok = min(r / G, n - 1), r_head = r - r / G * G;
  CodedRow<E, NF> mine[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i)
    if (i < heads) mine[i].ask(q + (size_t)(first + r_tok) * q_row_stride + (size_t)((g0 + i) * G + r_head) * D, D, col);

  // the blocks that the group's last token scores: all in front of its own, which are full
  const int scored = p0 + n - 1 < 0 ? 0 : (int)min((int64_t)((p0 + n - 1) >> 4), row_words);
  const int per_wg = phases * tiles_per_wave, tile0 = blockIdx.y * per_wg, tiles = (scored + 15) >> 4;
  if constexpr (kChoose) {
    const int seen = p0 < 0 ? 0 : scored + 1;
    if (seen <= to.K) {  // all of them
      int32_t* const out = to.blocks + ((int64_t)first * Hkv + g) * to.K;
      if (blockIdx.y == 0)
        for (int i = tid; i < to.K; i += kScoreThreads) out[i] = i < seen ? i : -1;
      return;
    }
  }
  if (tile0 >= tiles) return;

  // records of the wavefront's first tile and block ids of the second, on their way while the rows are coded
  const int32_t* const table = block_table + (size_t)b * bt_stride;
  const int tile_first = tile0 + phase, tile1 = min(tile0 + per_wg, tiles);
  auto block_at = [&](int tile) { return table[min(tile * 16 + col, scored - 1)]; };
  // (records two tiles ahead, block ids three)
  Records<NF> ahead[2];
  const int id0 = block_at(tile_first), id1 = block_at(tile_first + phases);
  int id2 = block_at(tile_first + 2 * phases);
  ahead[0].ask(codes, exponents, id0, g, Hkv, lane);
  ahead[1].ask(codes, exponents, id1, g, Hkv, lane);

#pragma unroll
  for (int i = 0; i < kHeads; ++i)
    if (i < heads) {
      const float scale_here = mine[i].code(&coded[i].row[r * kRow], col);
      if (col == 0) coded[i].scale[r] = scale_here;
    }
  __syncthreads();
  // operands of the rows: row r is head min(r % rows, G - 1) of token r / rows
  const int rows = 1 << log_rows;
  auto row_of = [&](int x) { return min(x >> log_rows, n - 1) * G + min(x & (rows - 1), G - 1); };
  i32x4 af[NF];
  float scale[4];
#pragma unroll
  for (int f = 0; f < NF; ++f) af[f] = *reinterpret_cast<const i32x4*>(&coded[here].row[row_of(col) * kRow + quad * 16 + f * 64]);
#pragma unroll
  for (int i = 0; i < 4; ++i) scale[i] = coded[here].scale[row_of(quad * 4 + i)];
  __syncthreads();  // (the tiles lie where the coded rows were)

  // scores of the group's first token from `out` on; lanes that hold none store behind the end, which the hardware leaves out
  float* const out = scores + ((int64_t)(first - t0) * Hkv + g) * row_words;
  const __amdgpu_buffer_rsrc_t to_scores = score_rows(out, n, Hkv, row_words);
  const int step = log_rows < 2 ? rows : 4;  // results 0, step, .. of a lane are tokens of their own
  int where[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = quad * 4 + i, tok = row >> log_rows;
    where[i] = (row & (rows - 1)) == 0 && tok < n ? (int)(tok * Hkv * row_words) * 4 + col * 4 : kNowhere;
  }
  char* const tile_lds = s_any + wave * Records<NF>::kBytes;
  auto walk = [&](Records<NF>& r, int tile) {
    r.put(tile_lds, lane);
    const int e = r.e;
    r.ask(codes, exponents, id2, g, Hkv, lane);  // (behind the last tile: its last block)
    id2 = block_at(tile + 3 * phases);
    i32x4 bf[NF], c = {0, 0, 0, 0};
    Records<NF>::get(bf, tile_lds, col, quad);
#pragma unroll
    for (int f = 0; f < NF; ++f) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(af[f], bf[f], c, 0, 0, 0);
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)c[i] * scale[i];
    // the maximum over a token's rows; it is then in v[0] (and, for one or two rows a token, v[2] or all four)
    if (log_rows >= 1) v[0] = fmaxf(v[0], v[1]), v[2] = fmaxf(v[2], v[3]);
    if (log_rows >= 2) v[0] = fmaxf(v[0], v[2]);
    if (log_rows >= 3) v[0] = max_of_rows16(v[0], v[0]);
    if (log_rows >= 4) v[0] = max_of_rows32(v[0], v[0]);
#pragma unroll
    for (int i = 0; i < (kChoose ? 1 : 4); ++i) {
      if (i & (step - 1)) continue;
      put_score<kChoose ? kAgent : 0>(to_scores, where[i], tile, v[i], e);
    }
  };
  for (int tile = tile_first; tile < tile1; tile += 2 * phases) {
    walk(ahead[0], tile);
    if (tile + phases >= tile1) break;
    walk(ahead[1], tile + phases);
  }
  if constexpr (kChoose) {
    const int wgs = (tiles + per_wg - 1) / per_wg;    // that score blocks of this row
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (this wavefront's scores are where every XCD finds them)
    __syncthreads();
    if (wgs > 1) {
      if (tid == 0) {
        uint32_t* const counter = counters + (int64_t)first * Hkv + g;
        s_order = (int)__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (s_order == wgs - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(s_order) != wgs - 1) return;
    }
    const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(out, 0, (int)row_words * 4, kRsrc);
    const int seen = scored + 1;
    choose<kScoreWaves, PER>([&](int j) { return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, j * 4, 0, kAgent)); }, wave, seen, to.keep_first,
                             seen - to.keep_last, to.K, to.blocks + ((int64_t)first * Hkv + g) * to.K, s_choose);
  }
}

// Rows (token, K/V head, head of the group padded to 1 << log_rows) of tokens from t0 on, as whole numbers; a row to each 16 lanes.
template <typename E, int NF>
__global__ __launch_bounds__(256) void code_kernel(const E* __restrict__ q, int q_row_stride, int8_t* __restrict__ coded, float* __restrict__ scale, int64_t rows,
                                                   int G, int log_rows, int Hkv, int D, int t0) {
  const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), at = min(r, rows - 1), pair = at >> log_rows, t = pair / Hkv;
  const int col = threadIdx.x & 15, h = min((int)(at & ((1 << log_rows) - 1)), G - 1), g = (int)(pair - t * Hkv);
  CodedRow<E, NF> mine;
  mine.ask(q + (size_t)(t0 + t) * q_row_stride + (size_t)(g * G + h) * D, D, col);
  const float s = mine.code(coded + at * (NF * 64), col);  // (the last row, possibly several times: the same bytes)
  if (col == 0) scale[at] = s;
}

constexpr int kPromptTiles = 4;  // row tiles of a wavefront
// Tokens of a wavefront of score_prompt_kernel; a workgroup has four times as many.
constexpr int prompt_tokens(int log_rows) { return kPromptTiles * (16 >> log_rows); }

// Grid: K/V heads, runs of `run` times four block tiles, token groups from unit0 on as in score_step_kernel.  The wavefronts of a workgroup have different tokens of the
// group; four tiles of blocks at a time, each brought in by one of them, serve all.  (Two workgroups per CU at least: of at most 256 registers the products' results are in those
// that other instructions can read; head sizes above 224 would spill for that: 512 tokens, 8 heads on 1 of 256, 20000 before them 33.5 us so, 26.1 with one.)
template <int NF, int LOG>
__global__ __launch_bounds__(kScoreThreads, NF < 8 ? 2 : 1) void score_prompt_kernel(const int8_t* __restrict__ coded, const float* __restrict__ scales,
                                                                      const int8_t* __restrict__ codes, const int8_t* __restrict__ exponents, Tokens tk,
                                                                      const int32_t* __restrict__ block_table, int bt_stride, float* __restrict__ scores,
                                                                      int64_t row_words, int Hkv, int unit0, int t0, int t1, int run) {
  constexpr int Dp = NF * 32, NA = kPromptTiles, kTokens = prompt_tokens(LOG), kGroup = kTokens * kScoreWaves, kPerTile = 16 >> LOG;
  __shared__ __attribute__((aligned(16))) char s_tiles[2][kScoreWaves][Records<NF>::kBytes];
  __shared__ int s_e[2][kScoreWaves][16];
  const int g = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
  const int unit = unit0 + blockIdx.z;
  auto first_unit = [&](int cu, int s) { return (long long)(cu / kGroup) + s; };
  const SeqOf seq = find_sequence(tk.cu_q, tk.ctx_before, tk.B, unit, first_unit);
  const int i0 = (int)(unit - first_unit(seq.tok0, seq.b)) * kGroup;
  const int group0 = max(seq.tok0 + i0, t0), in_group = min(min(seq.tok0 + i0 + kGroup, seq.tok0 + seq.S), t1) - group0;
  const int p_last = seq.cb + group0 - seq.tok0 + in_group - 1;
  if (in_group <= 0 || p_last < 0) return;
  // the blocks that the group's last token scores, the workgroup's share of them, and this wavefront's tokens (maybe none)
  const int scored = (int)min((int64_t)(p_last >> 4), row_words), tiles = (scored + 15) >> 4;
  const int super0 = blockIdx.y * run, super1 = min(super0 + run, (tiles + 3) >> 2);
  if (super0 >= super1) return;
  const int first = group0 + wave * kTokens, n = min(kTokens, in_group - wave * kTokens);

  i32x4 af[NA][NF];
  float scale[NA][4];
#pragma unroll
  for (int a = 0; a < NA; ++a) {
    auto row_of = [&](int x) { return (((int64_t)((n > 0 ? first : group0) - t0 + max(0, min(a * kPerTile + (x >> LOG), n - 1))) * Hkv + g) << LOG) + (x & ((1 << LOG) - 1)); };
    const int8_t* const row = coded + row_of(col) * (2 * Dp) + quad * 16;
#pragma unroll
    for (int f = 0; f < NF; ++f) af[a][f] = *reinterpret_cast<const i32x4*>(row + f * 64);
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[a][i] = scales[row_of(quad * 4 + i)];
  }
  const int32_t* const table = block_table + (size_t)seq.b * bt_stride;
  auto block_at = [&](int super) { return table[min((super * 4 + wave) * 16 + col, scored - 1)]; };
  Records<NF> ahead;
  ahead.ask(codes, exponents, block_at(super0), g, Hkv, lane);
  int id = block_at(super0 + 1);
  const __amdgpu_buffer_rsrc_t to_scores = score_rows(scores + ((int64_t)(first - t0) * Hkv + g) * row_words, max(n, 1), Hkv, row_words);
  // tokens whose results a lane stores: of each row tile all four, two or one, or, where the rows of lanes hold copies, of one tile in two or four
  constexpr int kPerRowTile = LOG == 0 ? 4 : LOG == 1 ? 2 : 1, kStores = LOG <= 2 ? NA * kPerRowTile : LOG == 3 ? NA / 2 : NA / 4;
  int where[kStores];
#pragma unroll
  for (int i = 0; i < kStores; ++i) {
    const int tok = LOG == 0   ? i / 4 * 16 + quad * 4 + i % 4
                    : LOG == 1 ? i / 2 * 8 + quad * 2 + i % 2
                    : LOG == 2 ? i * 4 + quad
                    : LOG == 3 ? (i * 2 + (quad & 1)) * 2 + (quad >> 1)
                               : i * 4 + quad;
    where[i] = tok < n ? (int)(tok * Hkv * row_words) * 4 + col * 4 : kNowhere;
  }
  auto put = [&](int i, float v, int e, int tile) { put_score<0>(to_scores, where[i], tile, v, e); };
  for (int super = super0; super < super1; ++super) {
    const int at = super & 1;
    ahead.put(s_tiles[at][wave], lane);
    if (lane < 16) s_e[at][wave][lane] = ahead.e;
    ahead.ask(codes, exponents, id, g, Hkv, lane);  // (behind the last one: its last block)
    id = block_at(super + 2);
    __syncthreads();  // (who has passed it has read the tiles before the last ones: one barrier a turn)
    if (n <= 0) continue;
#pragma unroll
    for (int k = 0; k < kScoreWaves; ++k) {
      const int tile = super * 4 + k, e = s_e[at][k][col];
      if (tile >= tiles) break;
      i32x4 bf[NF];
      Records<NF>::get(bf, s_tiles[at][k], col, quad);
      float m[NA];
#pragma unroll
      for (int a = 0; a < NA; ++a) {
        i32x4 c = {0, 0, 0, 0};
#pragma unroll
        for (int f = 0; f < NF; ++f) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(af[a][f], bf[f], c, 0, 0, 0);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)c[i] * scale[a][i];
        if constexpr (LOG == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) put(a * 4 + i, v[i], e, tile);
        } else if constexpr (LOG == 1) {
          put(a * 2, fmaxf(v[0], v[1]), e, tile);
          put(a * 2 + 1, fmaxf(v[2], v[3]), e, tile);
        } else {
          m[a] = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
          if constexpr (LOG == 2) put(a, m[a], e, tile);
        }
      }
      // a token's rows are in lanes of two (four) rows of lanes: two tiles change places in halves, and their maximum is the one's here, the other's there
      if constexpr (LOG == 3)
#pragma unroll
        for (int a = 0; a < NA; a += 2) put(a / 2, max_of_rows16(m[a], m[a + 1]), e, tile);
      if constexpr (LOG == 4) put(0, max_of_rows32(max_of_rows16(m[0], m[1]), max_of_rows16(m[2], m[3])), e, tile);
    }
  }
}

// A row to every WAVES wavefronts, rows (token, K/V head) from token t0 on.
template <int WAVES, int PER, int BINS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void choose_kernel(const float* __restrict__ scores, int64_t row_words, Tokens tk, Chosen to, int Hkv,
                                                                               int t0, int rows) {
  constexpr int kAtOnce = WAVES == 1 ? 4 : 1;  // rows of a workgroup
  __shared__ ChooseShared<WAVES, BINS> s[kAtOnce];
  const int of = WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x * kAtOnce + of, t = t0 + r / Hkv, tid = threadIdx.x - of * 64;
  if (r >= rows) return;
  int p;
  if (tk.cu_q) {
    const SeqOf seq = find_sequence(tk.cu_q, tk.ctx_before, tk.B, t, [](int cu, int) { return (long long)cu; });
    if (t - seq.tok0 >= seq.S) return;  // (behind the last sequence)
    p = seq.cb + t - seq.tok0;
  } else {
    p = tk.ctx_before[t];
  }
  const int n = p < 0 ? 0 : (int)min((int64_t)(p >> 4), row_words) + 1;
  int32_t* const out = to.blocks + ((int64_t)t0 * Hkv + r) * to.K;
  if (n <= to.K) {
    for (int i = tid; i < to.K; i += WAVES * 64) out[i] = i < n ? i : -1;
    return;
  }
  const float* const row = scores + (int64_t)r * row_words;
  choose<WAVES, PER>([&](int j) { return row[j]; }, wave, n, to.keep_first, n - to.keep_last, to.K, out, s[of]);
}

// Tokens [t0, t1) of a call, and what of it the launches need.
struct Slab {
  const SelectArgs& a;
  const Tokens tk;
  const int8_t *codes, *exponents;
  int64_t row_words;
  int log_rows, t0, t1;
  hipStream_t s;
  // tokens t of sequence b are in unit t / group + b or the one in front of it
  int unit0(int group) const { return a.cu_q ? std::max(0, t0 / group - 1) : t0; }
  int units(int group) const { return a.cu_q ? t1 / group + a.B + 1 - unit0(group) : t1 - t0; }
};

template <typename E, int NF, int PER>
void launch_step(const Slab& x) {
  const SelectArgs& a = x.a;
  const int group = a.cu_q ? 16 >> x.log_rows : 1, units = x.units(group), tiles = (int)(x.row_words / 16);
  // Up to four heads in a workgroup, a wavefront each: their records of a block are neighbours (32 sequences of 16384 to 131000 tokens, 8 heads of 128, both launches:
  // one head 84 us, four 76).  Where the workgroup also chooses, its wavefronts are at one row.
  const int log_heads = PER > 0 || a.Hkv % 2 != 0 ? 0 : a.Hkv % 4 != 0 ? 1 : 2, phases = kScoreWaves >> log_heads;
  // as many wavefronts as the device takes at once, then more tiles to one: up to 8 (the same call: 4 tiles 81 us, 8 76, 12 77)
  const int64_t waves = (int64_t)units * a.Hkv * tiles, room = (int64_t)a.num_cu * 32;
  const int most = std::max(8, tiles / (phases * 32768) + 1);  // (runs are a grid's second dimension)
  const int per_wave = (int)std::min<int64_t>(std::max<int64_t>(1, waves / room), most), runs = (tiles + phases * per_wave - 1) / (phases * per_wave);
  hipLaunchKernelGGL((score_step_kernel<E, NF, PER>), dim3((unsigned)(a.Hkv >> log_heads), (unsigned)runs, (unsigned)units), dim3(kScoreThreads), 0, x.s, (const E*)a.q,
                     a.q_row_stride, x.codes, x.exponents, x.tk, a.block_table, a.bt_stride, a.scores, x.row_words, a.Hq / a.Hkv, x.log_rows, a.Hkv, a.D, group,
                     x.unit0(group), x.t0, x.t1, per_wave, log_heads, Chosen{a.blocks, a.num_selected, a.keep_first, a.keep_last}, a.counters);
}

template <typename E, int NF>
void launch_prompts(const Slab& x) {
  const SelectArgs& a = x.a;
  const int64_t rows = ((int64_t)(x.t1 - x.t0) * a.Hkv) << x.log_rows;
  hipLaunchKernelGGL((code_kernel<E, NF>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, x.s, (const E*)a.q, a.q_row_stride, a.coded, a.scales, rows, a.Hq / a.Hkv,
                     x.log_rows, a.Hkv, a.D, x.t0);
  auto go = [&](auto log) {
    constexpr int LOG = decltype(log)::value, group = prompt_tokens(LOG) * kScoreWaves;
    const int units = x.units(group), tiles = (int)(x.row_words / 16);
    // four workgroups per CU; a workgroup walks eight tiles at least
    const int64_t wgs = ((int64_t)(x.t1 - x.t0) / group + 1) * a.Hkv;
    const int runs = (int)std::max<int64_t>(1, std::min<int64_t>((4 * a.num_cu + wgs - 1) / wgs, tiles / 8)), run = ((tiles + 3) / 4 + runs - 1) / runs;
    hipLaunchKernelGGL((score_prompt_kernel<NF, LOG>), dim3((unsigned)a.Hkv, (unsigned)(((tiles + 3) / 4 + run - 1) / run), (unsigned)units), dim3(kScoreThreads), 0, x.s, a.coded,
                       a.scales, x.codes, x.exponents, x.tk, a.block_table, a.bt_stride, a.scores, x.row_words, a.Hkv, x.unit0(group), x.t0, x.t1, run);
  };
  switch (x.log_rows) {
    case 0: return go(std::integral_constant<int, 0>());
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 3: return go(std::integral_constant<int, 3>());
    default: return go(std::integral_constant<int, 4>());
  }
}

template <typename E>
void launch_scores(const Slab& x, bool choose_too) {
  auto steps = [&](auto nf) {
    constexpr int NF = decltype(nf)::value;
    if (x.a.cu_q && x.a.T > 2 * x.a.B) launch_prompts<E, NF>(x);
    else if (choose_too) launch_step<E, NF, kFusedBlocks / kScoreThreads>(x);
    else launch_step<E, NF, 0>(x);
  };
  switch (summary_channels(x.a.D) / 32) {
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
  const Chosen to = {a.blocks, a.num_selected, a.keep_first, a.keep_last};
  const int64_t row_words = select_row_words(max_ctx_len);
  const int at_a_time = a.at_a_time;
  // (rows of no more blocks than are asked for, whatever the lengths: nothing is scored)
  const bool scored = row_words > a.num_selected, fused = scored && !a.cu_q && row_words <= kFusedBlocks;
  for (int t0 = 0; t0 < a.T; t0 += at_a_time) {
    const int t1 = std::min(a.T, t0 + at_a_time);
    const Slab x = {a, {a.cu_q, a.ctx_before, a.B, a.T}, codes, codes + summary_code_bytes(L), row_words, select_log_rows(L), t0, t1, s};
    if (scored) {
      if (L.dtype == ECOSERVE_BF16) launch_scores<uint16_t>(x, fused);
      else launch_scores<float>(x, fused);
    }
    if (fused) continue;
    const int rows = (t1 - t0) * a.Hkv;
    auto go = [&](auto kernel, int threads, int at_once) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(threads), 0, s, a.scores, row_words, x.tk, to, a.Hkv, t0, rows);
    };
    // A wavefront to a row, or, of few and of long rows, several (64 heads on 8, us of a call.  2048 blocks: 128 rows 19.5, with four 15.9, 2048 34.3 / 30.1, 8192 69.0 / 72.8; 6900
    // blocks, four / sixteen: 128 rows 23.6 / 21.6, 512 30.1 / 29.7, 1024 40.1 / 43.4, 4096 101 / 123).
    if (row_words <= 2048 && rows > 8 * a.num_cu) go(&choose_kernel<1, 32, 512>, 256, 4);
    else if (row_words <= 2048) go(&choose_kernel<4, 8, 1024>, 256, 1);
    else if (row_words <= 8192 && rows > 3 * a.num_cu) go(&choose_kernel<4, 32, 1024>, 256, 1);
    else if (row_words <= 8192) go(&choose_kernel<16, 8, 1024>, 1024, 1);
    else if (row_words <= 32768) go(&choose_kernel<16, 32, 1024>, 1024, 1);
    else go(&choose_kernel<16, 0, 1024>, 1024, 1);
  }
  return hipGetLastError();
}

}  // namespace eco
