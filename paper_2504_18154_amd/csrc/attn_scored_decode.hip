// Attention of one new token per sequence over the caches of ecoserve_cache, with formed scores, on gfx950 matrix cores.
//
// Eq. 2 of Section 2.1 for the decode phase, bound by the bytes of the cached keys and values (Table 2): 8-bit codes halve them.  A step is 64 tokens,
// four cache blocks, of one (sequence, K/V head); a wavefront loads a step straight into the operand layout of the matrix instructions, 16 bytes a lane and
// load, and decodes it in registers (a code is exact in bf16):
//   scores  S^T[token][head] = K . Q^T    v_mfma_f32_16x16x32_bf16, four tiles of 16 tokens; heads padded to 16 columns
//   values  O^T[d][head] += V^T . P^T     v_mfma_f32_16x16x32_bf16, twice 32 tokens
// A lane's load of V is a channel's 16 tokens of block `quad`, so its weights have to be those of the same tokens: row 4 q + i of tile t is token 4 t + i of
// block q, and P stays in registers.  Channels may go to the matrix instructions in any order that Q shares: a lane's 16 codes of K are two instructions'
// operands.  A scale belongs to a token: e4m3 keys take theirs in the conversion, int8 ones in the score; the values' multiply the weights.
// The registers of K are loaded again as soon as the step's scores are on their way, those of V behind the second product: a step is always in flight, and no
// second set of registers is needed.
//
// The steps of all (sequence, K/V head)s, head after head, and sequence after sequence, each with a few units in front that stand for the fixed cost of a piece, are
// one numbering, cut into equal shares, one per workgroup of a grid that the chip holds at once: whatever the lengths are (they live on the device, and every
// workgroup works the numbering out from them), all workgroups read as much and end together.  A share is the end of one (sequence, head), whole ones, and the
// beginning of another; a piece's steps are dealt in turn to the workgroup's wavefronts.  A piece that is a whole (sequence, head) writes the result; otherwise
// its state goes to the workspace, and the last workgroup of the (sequence, head) to arrive adds them up in the order of the keys.
//
// Weights are two bf16 numbers each, 16 bits, as in the other calls for a token over this cache; maxima, sums and the log-sum-exp are fp32, from the weights as they were.  The second parts
// ride in the eight columns that groups of up to eight heads leave (their columns repeat the heads, so a lane has both parts in hand and takes one), and cost a few vector instructions;
// larger groups take a product for each part (64 heads on 4 of 128, 32 x 16 k ... 131 k tokens over e4m3: 430 us, with weights of 8 bits 408; one of 20 000: 24.7 and 22.0).
//
// Measured: 32 contexts of 16 k ... 131 k tokens, 64 heads on 8 of 128, e4m3: 787 us (5.03 GB, 6.4 TB/s; reads reach 7.0).  64 of 100 ... 4000 tokens, 40 heads on 8: 58 us
// (4.2 TB/s: four of five heads are cut, a piece costs 5 us of latency, and its workgroup's neighbour on the CU covers half of it).  One of 20 000 tokens, int8: 20.9 us, of
// which 6 are the reads: the numbering, ids and first keys 6, the wavefronts' states 2, writing and counting 1.5, adding up 5.  96 windows of 1024 tokens, 8 heads on 1
// of 256, bf16: 31 us (3.2 TB/s), a workgroup to a CU.  Over codes, heads that do not fill an instance and capped or biased ones of 256 spill some 20 registers around the loop
// (32 x 9 k ... 60 k tokens, 8 heads of 80, int8: 4.5 TB/s).
//
// Lane layouts relied upon (lane = 16 quad + col), 16x16x32:  A[row = col][k = 8 quad .. + 7],  B[k = 8 quad .. + 7][col],  C[row = 4 quad + i][col].
#include <type_traits>

#include "quant.h"
#include "scored.h"
#include "softcap.h"

namespace eco {

namespace {

constexpr float kLowest = -3.0e38f;  // maximum before the first key: below every finite score, and no infinity to be subtracted from one
// The offset in the exponent is put this far above the largest score (log2 units), and again when one passes it: no weight is above 1, so that no sum leaves fp32 for the offset,
// and weights lose nothing by being small.
constexpr float kRoom = 8.f;
constexpr int kRsrc = 0x00020000;
constexpr int kAgent = 16;         // past the caches that XCDs do not share

__device__ const u32x4 kZeros[kBlockSize] = {};  // a unit of K of a block

template <int F, int NC>
struct Step {
  static constexpr bool kNarrow = F != kNative;
  // cache blocks of a step: two where the registers of bf16 heads of 256 allow no more (a lane then has half of a block's tokens)
  static constexpr int kBlocks = !kNarrow && NC == 8 ? 2 : 4, kTokens = 4 * kBlocks, kShift = kBlocks == 4 ? 6 : 5;
  static constexpr int NK = kNarrow ? NC / 2 : NC, NV = kNarrow ? 1 : kBlocks / 2;
  u32x4 k[kBlocks][NK];
  u32x4 v[2 * NC][NV];  // kTokens tokens of a channel
  u32x4 sk, sv;         // scales: e4m3: of the block whose keys the lane holds; otherwise as sv: of the block whose tokens it holds
};

__device__ __forceinline__ float across_quads_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float across_quads_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// A value that the compiler takes for new here: what is made of it is made here, and not kept in registers through the loops around.
__device__ __forceinline__ int here(int uniform) {
  asm volatile("" : "+s"(uniform));
  return uniform;
}
__device__ __forceinline__ int here_lane(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Words of dynamic LDS in front of the states: units before each sequence, and, of up to kHeldRanges of them, their ranges of keys.
constexpr int kHeldRanges = 1024;
__host__ __device__ constexpr int head_words(int B) { return ((B <= kHeldRanges ? 3 * B : B) + 1 + 3) / 4 * 4; }
// a / b for a >= 0, b > 0: 64 bits are rarely needed, and cost many times as much
__device__ __forceinline__ long long quotient(long long a, long long b) { return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b; }
// Channels whose states go through LDS at a time.
template <int NC>
constexpr int kPassChannels = NC == 8 ? 128 : 32 * NC;

// The states of all pieces of a (sequence, head), in order, as its result: by the last workgroup to arrive, all of it.  Piece 0's is the second state of its
// workgroup, the others' the first of theirs.  s_w [G][n_pieces], s_M, s_L [G], s_red [threads]: LDS.
template <int kWaves>
__device__ __forceinline__ void add_up(int tid, const float* first_state, int n_pieces, int G, int D, uint16_t* out_rows, float* lse_rows, float* s_w, float* s_M, float* s_L,
                                                 f32x4* s_red) {
  constexpr int kThreads = 64 * kWaves, kAtOnce = 4;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), state_words = scored_state_words(D);
  const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(first_state), 0, 2 * n_pieces * G * state_words * 4, kRsrc);
  auto state_at = [&](int k) { return (k == 0 ? 1 : 2 * k) * G * state_words; };  // in words
  // (groups of four channels; where the threads are more, several of them share a group's pieces.)
  const int groups = G * D / 4, parts = max(1, kThreads / groups);
  const int part = parts > 1 ? tid / groups : 0, i0 = parts > 1 ? tid - part * groups : tid;
  f32x4 x[kAtOnce];
  auto ask = [&](int i, int k0) {  // (behind the last piece: that one again, not added)
    const int h = i / (D / 4), at = h * state_words + 4 * (i - h * (D / 4));
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      x[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (state_at(min(k0 + j * parts, n_pieces - 1)) + at) * 4, 0, kAgent));
  };
  ask(min(i0, groups - 1), part);  // (the first ones: beside what says their weights)
  bool asked = true;
  for (int h = wave; h < G; h += kWaves) {
    constexpr int kMost = kScoredMostPieces / 64;
    float ms[kMost], ls[kMost], M = kLowest, L = 0.f;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      ms[i] = kLowest, ls[i] = 0.f;
      if (const int k = 64 * i + lane; k < n_pieces) {
        const u32x2 ml = __builtin_amdgcn_raw_buffer_load_b64(from, (state_at(k) + h * state_words + D) * 4, 0, kAgent);
        ms[i] = __uint_as_float(ml[0]);
        ls[i] = __uint_as_float(ml[1]);
      }
      M = fmaxf(M, ms[i]);
    }
    M = wave_max(M);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const float w = __builtin_amdgcn_exp2f(ms[i] - M);
      L += ls[i] * w;
      if (const int k = 64 * i + lane; k < n_pieces) s_w[h * n_pieces + k] = w;
    }
    L = wave_sum(L);
    if (lane == 0) s_M[h] = M, s_L[h] = L;
  }
  __syncthreads();
  for (int i = i0, turn = 0; parts > 1 ? turn == 0 : i < groups; i += kThreads, ++turn) {
    const bool here = part < parts && i < groups;
    const int h = here ? i / (D / 4) : 0, d = here ? 4 * (i - h * (D / 4)) : 0;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (here) {
      for (int k0 = part; k0 < n_pieces; k0 += kAtOnce * parts) {
        if (!asked) ask(i, k0);
        asked = false;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (k0 + j * parts < n_pieces) o += x[j] * s_w[h * n_pieces + k0 + j * parts];
      }
    }
    if (parts > 1) {
      s_red[tid] = o;
      __syncthreads();
      if (part == 0 && here)
        for (int p = 1; p < parts; ++p) o += s_red[p * groups + i];
    }
    if (part == 0 && here) {
      const float inv = 1.f / s_L[h];
      *reinterpret_cast<u32x2*>(out_rows + (size_t)h * D + d) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    }
  }
  if (lse_rows && tid < G) lse_rows[tid] = (s_M[tid] + log2f(s_L[tid])) * kLn2;
}

enum { kPlain, kFormed, kFarCapped };  // scores: scaled, capped (near: softcap.h) or with a bias or both, or capped far above them, with a bias or without

// Groups of up to kHalf heads: columns kHalf .. 2 kHalf - 1 of the products repeat the heads, and have the weights' second parts where the first columns have the first ones.
constexpr int kHalf = 8;

// kFull: the head vector fills the instance's channels.
// kWide: groups of more than kHalf heads, whose weights' parts are products of their own.
template <int F, int NC, int kForm, int kWaves, bool kFull, bool kWide>
__global__ __launch_bounds__(64 * kWaves, kWaves == 8 ? 2 : decode_scored_waves(F != kNative, NC, kWide)) void decode_scored_kernel(const uint16_t* __restrict__ q, int q_row_stride, const char* __restrict__ k_cache,
                                                                 const char* __restrict__ v_cache, const uint8_t* __restrict__ scales,
                                                                 const int32_t* __restrict__ block_table, int bt_stride, const int32_t* __restrict__ ctx_len,
                                                                 const int32_t* __restrict__ key_begin, const int32_t* __restrict__ key_end,
                                                                 const float* __restrict__ slopes, uint16_t* __restrict__ out, float* __restrict__ lse,
                                                                 float* states, uint32_t* counters, int B, int Hq, int Hkv, int G, int D, int num_cu,
                                                                 const Cap cap) {
  const float scale_log2e = cap.scale_log2e;
  constexpr int kThreads = 64 * kWaves;
  typedef Cached<F> C;
  typedef Step<F, NC> Frag;
  constexpr int kCh = kPassChannels<NC>, kRow = kCh + 4, kPasses = 32 * NC / kCh;
  extern __shared__ __attribute__((aligned(16))) uint32_t dynamic[];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16], s_M[16], s_L[16];
  __shared__ int s_sum[kWaves], s_most[kWaves], s_order;
  __shared__ f32x4 s_red[kThreads];
  int* const pre = reinterpret_cast<int*>(dynamic);  // [B + 1]: units of one K/V head before sequence b
  int* const key_lo = pre + B + 1;
  int* const key_hi = key_lo + B;
  float* const s_o = reinterpret_cast<float*>(dynamic) + head_words(B);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;

  // ---- the numbering
  const bool held = B <= kHeldRanges;
  auto range_of = [&](int b, int& lo, int& hi) {
    const int L = ctx_len[b];
    lo = key_begin ? max(key_begin[b], 0) : 0;
    hi = key_end ? min(key_end[b], L) : L;
  };
  auto steps_between = [](int lo, int hi) { return hi > lo ? ((hi - 1) >> Frag::kShift) - (lo >> Frag::kShift) + 1 : 0; };
  const int per = (B + kThreads - 1) / kThreads, b0 = tid * per;
  {
    int mine = 0, most = 0;
    for (int i = 0; i < per; ++i)
      if (const int b = b0 + i; b < B) {
        int lo, hi;
        range_of(b, lo, hi);
        if (held) key_lo[b] = lo, key_hi[b] = hi;
        const int n = steps_between(lo, hi);
        pre[b] = n + kPieceCost;
        mine += n + kPieceCost;
        most = max(most, n);
      }
    const int x = lanes_prefix_sum(mine);
    most = lanes_max(most);
    if (lane == 63) s_sum[wave] = x, s_most[wave] = most;
    __syncthreads();
    int run = x - mine;
    for (int w = 0; w < wave; ++w) run += s_sum[w];
    for (int i = 0; i < per; ++i)
      if (b0 + i < B) {
        const int n = pre[b0 + i];
        pre[b0 + i] = run;
        run += n;
        if (b0 + i == B - 1) pre[B] = run;
      }
  }
  int most = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = max(most, s_most[w]);
  __syncthreads();
  const int head_units = __builtin_amdgcn_readfirstlane(pre[B]);
  const long long units = (long long)head_units * Hkv;
  // a share; at least kLeastSteps, and as many as leave a (sequence, head) no more pieces than the last one to arrive has room for
  // (short ones: no more workgroups than CUs, since two on one CU would be the last to end)
  int share = (int)quotient(units + gridDim.x - 1, gridDim.x);
  if (share < kShortShare) share = (int)quotient(units + num_cu - 1, num_cu);
  share = max(max(kLeastSteps, share), __builtin_amdgcn_readfirstlane(most) / (kScoredMostPieces - 2) + 1);
  auto owner = [&](long long u) { return (int)quotient(u, share); };
  const int blk_bytes = kBlockSize * D * C::kBytes;                   // of a (block, head)
  const uint32_t blk_stride = (uint32_t)Hkv * (uint32_t)blk_bytes, scale_stride = (uint32_t)Hkv * kScaleBytes;
  auto at_block = [](int id, uint32_t stride) { return (size_t)(uint32_t)id * stride; };
  const int wg = blockIdx.x;
  long long u = (long long)wg * share;
  const long long u_end = min(units, u + share);
  if (u >= u_end) return;
  int g = (int)quotient(u, head_units), b;
  {
    const int at = (int)(u - (long long)g * head_units);
    int lo = 0, n_cand = B;  // the largest b with pre[b] <= at, 64 candidates at a time
    while (n_cand > 1) {
      const int stride = (n_cand + 63) >> 6, idx = lo + lane * stride;
      const bool le = idx < lo + n_cand && pre[min(idx, B)] <= at;
      const int next = lo + max((int)__popcll(__ballot(le)) - 1, 0) * stride;
      n_cand = min(stride, lo + n_cand - next);
      lo = next;
    }
    b = __builtin_amdgcn_readfirstlane(lo);
  }

  for (;; g = b + 1 == B ? g + 1 : g, b = b + 1 == B ? 0 : b + 1) {
    // ---- the next piece: steps [p0, p1) of the n of (b, g)
    const long long first_unit = (long long)g * head_units + __builtin_amdgcn_readfirstlane(pre[b]);
    if (first_unit >= u_end) break;
    const int n = __builtin_amdgcn_readfirstlane(pre[b + 1] - pre[b]) - kPieceCost;
    const int p0 = (int)max(u - first_unit - kPieceCost, 0LL), p1 = (int)min((long long)n, max(u_end - first_unit - kPieceCost, 0LL));
    uint16_t* const out_rows = out + ((size_t)b * Hq + (size_t)g * G) * D;
    float* const lse_rows = lse ? lse + (size_t)b * Hq + g * G : nullptr;
    if (n == 0 && u <= first_unit) {  // no keys
      for (int i = tid; i < G * D / 2; i += kThreads) reinterpret_cast<uint32_t*>(out_rows)[i] = 0;
      if (lse_rows && tid < G) lse_rows[tid] = -INFINITY;
    }
    if (p0 >= p1) continue;
    int lo, hi;
    if (held) lo = __builtin_amdgcn_readfirstlane(key_lo[b]), hi = __builtin_amdgcn_readfirstlane(key_hi[b]);
    else range_of(b, lo, hi);
    const int s_first = (lo >> Frag::kShift) + p0, count = p1 - p0 > wave ? (p1 - p0 - wave + kWaves - 1) / kWaves : 0;  // this wavefront's steps: s_first + wave + kWaves i
    const int first_wg = owner(first_unit + kPieceCost), n_pieces = owner(first_unit + kPieceCost + n - 1) - first_wg + 1;

    // ---- query rows: B operand, channels in the order of the keys' units
    bf16x8 qf[NC];
    {
      const int l_ = here_lane(lane), col_ = l_ & (kWide ? 15 : kHalf - 1), quad_ = l_ >> 4, D_ = here(D);
      const uint16_t* const q_row = q + (size_t)b * q_row_stride + ((size_t)g * G + col_) * D_;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int d = Frag::kNarrow ? 64 * (c >> 1) + 16 * quad_ + 8 * (c & 1) : 32 * c + 8 * quad_;
        const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
        qf[c] = col_ < G && d < D_ ? *reinterpret_cast<const bf16x8*>(q_row + d) : zero;
      }
    }
    float slope = 0.f;
    int position = 0;
    if (kForm != kPlain && slopes) {
      position = ctx_len[b] - 1;
      if (const int h = kWide ? col : col & (kHalf - 1); h < G) slope = slopes[g * G + h] * kLog2e;
    }

    // ---- loads
    const int32_t* const table = block_table + (size_t)b * bt_stride;
    const int blk_lo = lo >> 4, blk_hi = (hi - 1) >> 4;
    constexpr int kBlocks = Frag::kBlocks;
    // row 4 c + i of tile t, and what lane quad c holds, is token slot_of(c) + 4 t + i of block block_of(c)
    auto block_of = [](int c) { return kBlocks == 4 ? c : c >> 1; };
    auto slot_of = [](int c) { return kBlocks == 4 ? 0 : 8 * (c & 1); };
    // the block of this wavefront's step i that lane quad c has to do with: the only ones named are those that hold keys of the range
    auto block_id = [&](int i, int c) { return table[min(max(kBlocks * (s_first + wave + kWaves * i) + block_of(c), blk_lo), blk_hi)]; };
    const char* const k_head = k_cache + (size_t)g * blk_bytes + (slot_of(col >> 2) + (col & 3)) * 16;
    const char* const v_head = v_cache + (size_t)g * blk_bytes + (col * kBlockSize + slot_of(quad)) * C::kBytes;
    const uint8_t* const s_head = Frag::kNarrow ? scales + (size_t)g * kScaleBytes : nullptr;
    auto load_k = [&](Frag& f, int id) {
      const char* const at = k_head + at_block(id, blk_stride);
#pragma unroll
      for (int j = 0; j < Frag::NK; ++j) {
        // (behind the head vector, where Q is zero: codes of its first unit, which are finite, and zeros in the place of elements, which may not be)
        const int unit = 4 * j + quad;
        const bool there = kFull || unit * C::kUnit < D;
        const char* const unit_at = Frag::kNarrow || there ? at + (there ? unit : 0) * 256 : reinterpret_cast<const char*>(kZeros);
#pragma unroll
        for (int t = 0; t < kBlocks; ++t) f.k[t][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(unit_at + 64 * t));
      }
      if constexpr (F == kE4m3) f.sk = *reinterpret_cast<const u32x4*>(s_head + at_block(id, scale_stride));
    };
    auto load_v = [&](Frag& f, int id) {
      const char* const at = v_head + at_block(id, blk_stride);
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt)
        if (kFull || 16 * dt < D)
#pragma unroll
          for (int h = 0; h < Frag::NV; ++h) f.v[dt][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + dt * 256 * C::kBytes + 16 * h));
      if constexpr (Frag::kNarrow) {
        const uint8_t* const sc = s_head + at_block(id, scale_stride);
        f.sv = *reinterpret_cast<const u32x4*>(sc + kBlockSize);
        if constexpr (F == kInt8) f.sk = *reinterpret_cast<const u32x4*>(sc);
      }
    };
    int next_k = 0, next_v = 0;  // the next step's, asked for a step ahead

    // ---- a step
    f32x4 acc[2 * NC];
#pragma unroll
    for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kLowest, l = 0.f;
    // (edges: the range may begin or end within the step)
    auto process = [&](Frag& f, int i, auto more, auto edges) {
      constexpr bool kEdge = decltype(edges)::value;
      constexpr int kTokens = Frag::kTokens;
      constexpr bool kOpen = !Frag::kNarrow;
      const int k0 = (s_first + wave + kWaves * i) << Frag::kShift;
      f32x4 s[kBlocks];
#pragma unroll
      for (int t = 0; t < kBlocks; ++t) {
        if (Frag::kNarrow) __builtin_amdgcn_sched_barrier(0);  // (decoded operands are made when they are due: together they would need twice the registers of the codes)
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float k_scale = F == kE4m3 ? scale_of_byte((f.sk[t] >> (8 * (col & 3))) & 255u) : 1.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          bf16x8 a;
          if constexpr (Frag::kNarrow) a = codes_to_bf16x8<F>(f.k[t][c >> 1][2 * (c & 1)], f.k[t][c >> 1][2 * (c & 1) + 1], k_scale);
          else a = __builtin_bit_cast(bf16x8, f.k[t][c]);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[c], s[t], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (decltype(more)::value) load_k(f, next_k);
      // Keys outside the range (stale slots, tokens that a window has passed): their scores are excluded and what stands in their place is
      // cleared, since 0 times a stale NaN would reach the sums.
      [[maybe_unused]] const int lane0 = k0 + 16 * block_of(quad) + slot_of(quad), first = lo - lane0, last = hi - lane0;  // token j of the lane's is in sight: first <= j < last
      if constexpr (kEdge) {
        auto keep = [&](int j, uint32_t bits) { return j >= first && j < last ? bits : 0u; };
        if constexpr (Frag::kNarrow) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t bytes = keep(4 * w, 0xffu) | keep(4 * w + 1, 0xff00u) | keep(4 * w + 2, 0xff0000u) | keep(4 * w + 3, 0xff000000u);
            f.sv[w] &= bytes;
#pragma unroll
            for (int dt = 0; dt < 2 * NC; ++dt) f.v[dt][0][w] &= bytes;
          }
        } else {
#pragma unroll
          for (int w = 0; w < kTokens / 2; ++w) {
            const uint32_t halves = keep(2 * w, 0xffffu) | keep(2 * w + 1, 0xffff0000u);
#pragma unroll
            for (int dt = 0; dt < 2 * NC; ++dt) f.v[dt][w >> 2][w & 3] &= halves;
          }
        }
      }
      float x[kTokens];
#pragma unroll
      for (int j = 0; j < kTokens; ++j) x[j] = s[j >> 2][j & 3];
      [[maybe_unused]] auto scaled = [&](const u32x4& by) {
#pragma unroll
        for (int w = 0; w < kTokens / 4; ++w) x[4 * w] *= scale_of<0>(by[w]), x[4 * w + 1] *= scale_of<1>(by[w]), x[4 * w + 2] *= scale_of<2>(by[w]), x[4 * w + 3] *= scale_of<3>(by[w]);
      };
      if constexpr (F == kInt8) scaled(f.sk);
      if constexpr (kForm != kPlain) {
        if constexpr (kForm == kFarCapped) {
#pragma unroll
          for (int j = 0; j < kTokens; ++j) x[j] = far_cap(x[j], cap);
        } else if (cap.kind == kNear) {
#pragma unroll
          for (int j = 0; j < kTokens; ++j) x[j] = __builtin_fmaf(2.f * cap.log2e, near_cap(x[j], cap), cap.log2e);
        } else {
#pragma unroll
          for (int j = 0; j < kTokens; ++j) x[j] *= scale_log2e;
        }
        if (slopes) {
          const int away = lane0 - position;
#pragma unroll
          for (int j = 0; j < kTokens; ++j) x[j] = __builtin_fmaf(slope, (float)(away + j), x[j]);
        }
      }
      if constexpr (kEdge) {
#pragma unroll
        for (int j = 0; j < kTokens; ++j)
          if (j < first || j >= last) x[j] = -INFINITY;
      }
      const float c = kForm != kPlain ? 1.f : scale_log2e;  // (formed scores are in the exp2 domain already)
      float top = max3(x[0], x[1], x[2]);
#pragma unroll
      for (int j = 3; j < kTokens - 1; j += 2) top = max3(top, x[j], x[j + 1]);
      top = across_quads_max(fmaxf(top, x[kTokens - 1])) * c;
      if (__any(top > m)) {
        const float m_new = top > m ? top + kRoom : m, alpha = __builtin_amdgcn_exp2f(m - m_new);
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] *= alpha;
        m = m_new;
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kTokens; ++j) {
        x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], c, -m));
        sum[j & 1] += x[j];
      }
      l += sum[0] + sum[1];
      if constexpr (Frag::kNarrow) scaled(f.sv);
#pragma unroll
      for (int h = 0; h < kBlocks / 2; ++h) {
        u32x4 high, low;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float &a = x[8 * h + 2 * i], &b = x[8 * h + 2 * i + 1];
          high[i] = first_parts<kOpen>(a, b);
          if constexpr (kWide) {
            low[i] = second_parts<kOpen>(a, b, high[i]);
          } else {
            // (the columns' mask is made here: held through the loop, or with both parts made before one is taken, registers spilled: 64 x 100 ... 4000 tokens 74 us for 57)
            const uint32_t second = (uint32_t)((here_lane(lane) << 28) >> 31);
            if constexpr (kOpen) {
              high[i] = second ? second_parts<kOpen>(a, b, high[i]) : high[i];
            } else {
              a -= __uint_as_float(high[i] << 16 & second), b -= __uint_as_float(high[i] & 0xffff0000u & second);
              high[i] = pack_bf16x2(a, b);
            }
          }
        }
#pragma unroll
        for (int dt = 0; dt < 2 * NC; ++dt) {
          if (Frag::kNarrow && dt % 2 == 0) __builtin_amdgcn_sched_barrier(0);
          bf16x8 a;
          if constexpr (Frag::kNarrow) a = codes_to_bf16x8<F>(f.v[dt][0][2 * h], f.v[dt][0][2 * h + 1], 1.f);
          else a = __builtin_bit_cast(bf16x8, f.v[dt][h % Frag::NV]);
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, high), acc[dt], 0, 0, 0);
          if constexpr (kWide) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, low), acc[dt], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (decltype(more)::value) {
        load_v(f, next_v);
        next_k = block_id(i + 2, col >> 2);
        next_v = block_id(i + 2, quad);
      }
    };
    if (count > 0) {
      // a first step that the range begins in comes last, beside the one that it may end in
      const bool late = count > 1 && (s_first + wave) << Frag::kShift < lo;
      Frag f;
      load_k(f, block_id(late, col >> 2));
      load_v(f, block_id(late, quad));
      next_k = block_id(late + 1, col >> 2);
      next_v = block_id(late + 1, quad);
      for (int i = late; i < count - 1; ++i) process(f, i, std::true_type(), std::false_type());
      for (int i = count - 1;;) {
        process(f, i, std::false_type(), std::true_type());
        if (!late || i == 0) break;
        i = 0;
        load_k(f, block_id(0, col >> 2));
        load_v(f, block_id(0, quad));
      }
    }

    // ---- the wavefronts' states, added up
    // (what is worked out from the thread's number from here on is not kept through the loop over the keys)
    const int tid_ = here_lane(tid), col_ = tid_ & 15, quad_ = (tid_ >> 4) & 3, D_ = here(D), G_ = here(G), words_ = scored_state_words(D_);
    l = across_quads_sum(l);
    if (quad_ == 0) s_m[wave][col_] = m, s_l[wave][col_] = l;
    __syncthreads();
    {
      float M = s_m[0][col_];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][col_]);
      const float alpha = __builtin_amdgcn_exp2f(m - M);
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] *= alpha;
      if (wave == 0 && quad_ == 0) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += s_l[w][col_] * __builtin_amdgcn_exp2f(s_m[w][col_] - M);
        s_M[col_] = M;
        s_L[col_] = sum;
      }
    }
    if constexpr (!kWide) {
      // the weights' second parts
      auto turned = [](float x) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, true)); };  // row_ror:8
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[dt][i] += turned(acc[dt][i]);
    }
    // (a workgroup has two states at most: of the piece that it ends, and of the one that it begins and does not end)
    float* const state = states + (size_t)(2 * wg + (p0 == 0 ? 1 : 0)) * G_ * words_;
    const __amdgpu_buffer_rsrc_t to_state = __builtin_amdgcn_make_buffer_rsrc(state, 0, G_ * words_ * 4, kRsrc);
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      if (pass > 0) __syncthreads();
      if (col_ < G_)
#pragma unroll
        for (int dt = 0; dt < kCh / 16; ++dt)
          *reinterpret_cast<f32x4*>(s_o + ((size_t)wave * G_ + col_) * kRow + 16 * dt + 4 * quad_) = acc[pass * (kCh / 16) + dt];
      __syncthreads();
      for (int i = tid_; i < G_ * (kCh / 4); i += kThreads) {
        const int h = i / (kCh / 4), at = 4 * (i % (kCh / 4)), d = pass * kCh + at;
        if (d >= D_) continue;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o += *reinterpret_cast<const f32x4*>(s_o + ((size_t)w * G_ + h) * kRow + at);
        if (n_pieces == 1) {
          const float inv = 1.f / s_L[h];
          *reinterpret_cast<u32x2*>(out_rows + (size_t)h * D_ + d) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        } else {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), to_state, (h * words_ + d) * 4, 0, kAgent);
        }
      }
    }
    if (n_pieces == 1) {
      if (lse_rows && tid_ < G_) lse_rows[tid_] = (s_M[tid_] + log2f(s_L[tid_])) * kLn2;
      __syncthreads();
      continue;
    }
    if (tid_ < G_)
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(s_M[tid_]), __float_as_uint(s_L[tid_])}, to_state, (tid_ * words_ + D_) * 4, 0, kAgent);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid_ == 0) s_order = (int)atomicInc(counters + (size_t)b * Hkv + g, (unsigned)n_pieces - 1);  // (the last one wraps it to zero)
    __syncthreads();
    if (s_order != n_pieces - 1) continue;  // (s_order is written again behind two barriers at least)

    add_up<kWaves>(tid_, states + (size_t)2 * first_wg * G_ * words_, n_pieces, G_, D_, out_rows, lse_rows, s_o, s_M, s_L, s_red);
    __syncthreads();
  }
}

template <int F, int NC, int kWaves, bool kWide>
void launch_waves(const ScoredArgs& a, hipStream_t s) {
  const int G = a.Hq / a.Hkv;
  const Cap cap = make_cap(a.softcap, a.scale_log2e);
  // states of the wavefronts, or the weights of the pieces when they are added up
  const size_t words = std::max((size_t)kWaves * G * (kPassChannels<NC> + 4), (size_t)G * kScoredMostPieces);
  const size_t lds = (head_words(a.B) + words) * sizeof(uint32_t);
  const int grid = (kWaves == 8 ? 1 : decode_scored_waves(F != kNative, NC, kWide)) * a.num_cu;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * kWaves), lds, s, (const uint16_t*)a.q, a.q_row_stride, (const char*)a.k_cache, (const char*)a.v_cache, a.scales,
                       a.block_table, a.bt_stride, a.ctx_before, a.key_begin, a.key_end, a.slopes, (uint16_t*)a.out, a.lse, a.states, a.counters, a.B, a.Hq, a.Hkv, G,
                       a.D, a.num_cu, cap);
  };
  const bool full = a.D == 32 * NC;
  auto with_form = [&](auto kind) {
    constexpr int kForm = decltype(kind)::value;
    full && !kWide ? go(&decode_scored_kernel<F, NC, kForm, kWaves, !kWide, kWide>) : go(&decode_scored_kernel<F, NC, kForm, kWaves, false, kWide>);
  };
  if (cap.kind == kFar) with_form(std::integral_constant<int, kFarCapped>());
  else if (cap.kind == kNear || a.slopes) with_form(std::integral_constant<int, kFormed>());
  else with_form(std::integral_constant<int, kPlain>());
}
template <int F, int NC>
void launch_formed(const ScoredArgs& a, hipStream_t s) {
  const bool wide = a.Hq / a.Hkv > kHalf;
  if constexpr (F != kNative && NC <= 4) {
    if (decode_scored_short((int64_t)a.B * a.Hkv * ((a.max_ctx_len + 63) / 64 + kPieceCost), true, NC, a.num_cu)) return wide ? launch_waves<F, NC, 8, true>(a, s) : launch_waves<F, NC, 8, false>(a, s);
  }
  wide ? launch_waves<F, NC, 4, true>(a, s) : launch_waves<F, NC, 4, false>(a, s);
}

template <int F>
void launch_format(const ScoredArgs& a, hipStream_t s) {
  switch (scored_chunks(a.D)) {
    case 2: return launch_formed<F, 2>(a, s);
    case 4: return launch_formed<F, 4>(a, s);
    default: return launch_formed<F, 8>(a, s);
  }
}

}  // namespace

hipError_t launch_decode_scored(const ScoredArgs& a, hipStream_t s) {
  switch (a.format) {
    case kInt8: launch_format<kInt8>(a, s); break;
    case kE4m3: launch_format<kE4m3>(a, s); break;
    default: launch_format<kNative>(a, s); break;
  }
  return hipGetLastError();
}

}  // namespace eco
