// Attention of one new token per sequence over the caches of ecoserve_cache, with formed scores, on gfx950 matrix cores.
//
// Eq. 2 of Section 2.1 for the decode phase, bound by the bytes of the cached keys and values (Table 2): 8-bit codes halve them.  A step is 32 tokens,
// two cache blocks, of one (sequence, K/V head); a wavefront loads a step straight into the operand layout of the matrix instructions and decodes it in
// registers (a code is exact in bf16), 4 KiB of K and 4 KiB of V for D = 128:
//   scores  S^T[token][head] = K . Q^T    v_mfma_f32_16x16x32_bf16, two tiles of 16 tokens; heads padded to 16 columns
//   values  O^T[d][head] += V^T . P^T     v_mfma_f32_16x16x32_bf16 over the step's 32 tokens
// Row r = 4 q + i of tile t is token 8 q + 4 t + i of the step, so the scores that a lane holds after both tiles are those of 8 neighbouring tokens, which is
// the B operand of the second product: P stays in registers.  A scale belongs to a token, so the keys' scales multiply scores and the values' weights.
// Channels may go to the matrix instructions in any order that Q shares: a lane's 16 codes of a unit are two instructions' operands.
//
// The steps of all (sequence, K/V head)s are cut into slices of about equal length, which every workgroup works out from the lengths (they live on the
// device): a slice at a time is dealt to the workgroups of a grid of three per CU, its steps in turn to the workgroup's four wavefronts.  A slice that is a
// whole (sequence, head) writes the result; otherwise its state goes to the workspace and the last workgroup of the (sequence, head) to arrive adds them up
// in order, whichever comes last.
//
// Weights are rounded to bf16 for the second product (2^-9 of each, unbiased: the result's own rounding is as large); maxima, sums and the
// log-sum-exp are fp32, from the weights before that rounding.
//
// Lane layouts relied upon (lane = 16 quad + col), 16x16x32:  A[row = col][k = 8 quad .. + 7],  B[k = 8 quad .. + 7][col],  C[row = 4 quad + i][col].
#include <type_traits>

#include "quant.h"
#include "scored.h"

namespace eco {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kLeastSteps = 16;    // of a slice that is not the last of its sequence's equal parts
constexpr float kLowest = -3.0e38f;  // maximum before the first key: below every finite score, and no infinity to be subtracted from one
constexpr float kTau = 8.f;        // the maximum in the exponent is raised when a score passes it by 2^8: weights reach that, and lose nothing by it
constexpr int kRsrc = 0x00020000;
constexpr int kAgent = 16;         // past the caches that XCDs do not share

template <int F, int NC>
struct Step {
  static constexpr bool kNarrow = F != kNative;
  static constexpr int NK = kNarrow ? NC / 2 : NC;
  typedef typename std::conditional<kNarrow, u32x2, u32x4>::type VReg;
  u32x4 k[2][NK];
  VReg v[2 * NC];
  u32x2 sk, sv;
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

// Words of dynamic LDS in front of the states: slices before each sequence, and, of up to kHeldRanges of them, their ranges of keys.
constexpr int kHeldRanges = 1024;
__host__ __device__ constexpr int head_words(int B) { return ((B <= kHeldRanges ? 3 * B : B) + 1 + 3) / 4 * 4; }
// Channels whose states go through LDS at a time.
template <int NC>
constexpr int kPassChannels = NC == 8 ? 128 : 32 * NC;

template <int F, int NC, bool kForm>
__global__ __launch_bounds__(kThreads, NC == 8 ? 1 : 2) void decode_scored_kernel(const uint16_t* __restrict__ q, int q_row_stride, const char* __restrict__ k_cache,
                                                                 const char* __restrict__ v_cache, const uint8_t* __restrict__ scales,
                                                                 const int32_t* __restrict__ block_table, int bt_stride, const int32_t* __restrict__ ctx_len,
                                                                 const int32_t* __restrict__ key_begin, const int32_t* __restrict__ key_end,
                                                                 const float* __restrict__ slopes, uint16_t* __restrict__ out, float* __restrict__ lse,
                                                                 float* states, uint32_t* counters, int B, int Hq, int Hkv, int G, int D, int want,
                                                                 float scale_log2e, float cap_in, float cap_log2e) {
  typedef Cached<F> C;
  typedef Step<F, NC> Frag;
  constexpr int kCh = kPassChannels<NC>, kRow = kCh + 4, kPasses = 32 * NC / kCh;
  extern __shared__ __attribute__((aligned(16))) uint32_t dynamic[];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16], s_M[16], s_L[16];
  __shared__ long long s_sum[kWaves];
  __shared__ int s_scan[kWaves], s_order;
  __shared__ f32x4 s_red[kThreads];
  uint32_t* const pre = dynamic;  // [B + 1]: low half: slices of one K/V head before sequence b; high half: those of sequences that are cut
  int* const key_lo = reinterpret_cast<int*>(dynamic) + B + 1;
  int* const key_hi = key_lo + B;
  float* const s_o = reinterpret_cast<float*>(dynamic) + head_words(B);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;

  // ---- slices
  const bool held = B <= kHeldRanges;
  auto range_of = [&](int b, int& lo, int& hi) {
    const int L = ctx_len[b];
    lo = key_begin ? max(key_begin[b], 0) : 0;
    hi = key_end ? min(key_end[b], L) : L;
  };
  auto steps_between = [](int lo, int hi) { return hi > lo ? ((hi - 1) >> 5) - (lo >> 5) + 1 : 0; };
  auto steps_of = [&](int b) {
    int lo, hi;
    if (held) lo = key_lo[b], hi = key_hi[b];
    else range_of(b, lo, hi);
    return steps_between(lo, hi);
  };
  const int per = (B + kThreads - 1) / kThreads, b0 = tid * per;
  {
    long long mine = 0;
    for (int i = 0; i < per; ++i)
      if (const int b = b0 + i; b < B) {
        int lo, hi;
        range_of(b, lo, hi);
        if (held) key_lo[b] = lo, key_hi[b] = hi;
        mine += steps_between(lo, hi);
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
    if (lane == 0) s_sum[wave] = mine;
  }
  __syncthreads();
  const long long all = (s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]) * Hkv, even = (all + want - 1) / want;
  const int length = (int)max((long long)kLeastSteps, min(even, 1LL << 30));
  auto slices_of = [&](int n) { return n <= length ? 1 : min((n + length - 1) / length, kScoredMostSlices); };
  {
    uint32_t mine = 0;
    for (int i = 0; i < per; ++i)
      if (b0 + i < B) {
        const uint32_t n = slices_of(steps_of(b0 + i));
        mine += n + (n > 1 ? n << 16 : 0u);
      }
    const int x = lanes_prefix_sum((int)mine);
    if (lane == 63) s_scan[wave] = x;
    __syncthreads();
    uint32_t run = (uint32_t)x - mine;
    for (int w = 0; w < wave; ++w) run += (uint32_t)s_scan[w];
    for (int i = 0; i < per; ++i)
      if (b0 + i < B) {
        pre[b0 + i] = run;
        const uint32_t n = slices_of(steps_of(b0 + i));
        run += n + (n > 1 ? n << 16 : 0u);
        if (b0 + i == B - 1) pre[B] = run;
      }
  }
  __syncthreads();
  const int items = (int)(pre[B] & 0xffffu) * Hkv;
  const int blk_bytes = kBlockSize * D * C::kBytes;                   // of a (block, head)
  const long long blk_stride = (long long)Hkv * blk_bytes;
  const int state_words = scored_state_words(D);

  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int slice = item / Hkv, g = item - slice * Hkv;
    int b;
    {
      int lo = 0, n_cand = B;
      while (n_cand > 1) {
        const int stride = (n_cand + 63) >> 6, idx = lo + lane * stride;
        const bool le = idx < lo + n_cand && (int)(pre[min(idx, B)] & 0xffffu) <= slice;
        const int next = lo + max((int)__popcll(__ballot(le)) - 1, 0) * stride;
        n_cand = min(stride, lo + n_cand - next);
        lo = next;
      }
      b = __builtin_amdgcn_readfirstlane(lo);
    }
    const uint32_t from = pre[b], to = pre[b + 1];
    const int k_slice = __builtin_amdgcn_readfirstlane(slice - (int)(from & 0xffffu)), n_slices = __builtin_amdgcn_readfirstlane((int)(to & 0xffffu) - (int)(from & 0xffffu));
    int lo, hi;
    if (held) lo = __builtin_amdgcn_readfirstlane(key_lo[b]), hi = __builtin_amdgcn_readfirstlane(key_hi[b]);
    else range_of(b, lo, hi);
    const int n = steps_between(lo, hi);
    uint16_t* const out_rows = out + ((size_t)b * Hq + (size_t)g * G) * D;
    float* const lse_rows = lse ? lse + (size_t)b * Hq + g * G : nullptr;
    if (n == 0) {  // no keys
      for (int i = tid; i < G * D / 2; i += kThreads) reinterpret_cast<uint32_t*>(out_rows)[i] = 0;
      if (lse_rows && tid < G) lse_rows[tid] = -INFINITY;
      continue;
    }
    const int s_first = __builtin_amdgcn_readfirstlane((lo >> 5) + (int)((long long)n * k_slice / n_slices));
    const int s_last = __builtin_amdgcn_readfirstlane((lo >> 5) + (int)((long long)n * (k_slice + 1) / n_slices));
    const int count = s_last - s_first > wave ? (s_last - s_first - wave + kWaves - 1) / kWaves : 0;  // this wavefront's steps: s_first + wave + 4 i

    // ---- query rows: B operand, channels in the order of the keys' units
    bf16x8 qf[NC];
    const uint16_t* const q_row = q + (size_t)b * q_row_stride + ((size_t)g * G + col) * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int d = Frag::kNarrow ? 64 * (c >> 1) + 16 * quad + 8 * (c & 1) : 32 * c + 8 * quad;
      const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
      qf[c] = col < G && d < D ? *reinterpret_cast<const bf16x8*>(q_row + d) : zero;
    }
    float slope = 0.f;
    int position = 0;
    if (kForm && slopes) {
      position = ctx_len[b] - 1;
      if (col < G) slope = slopes[g * G + col] * kLog2e;
    }

    // ---- loads
    const int32_t* const table = block_table + (size_t)b * bt_stride;
    const int blk_lo = lo >> 4, blk_hi = (hi - 1) >> 4;
    auto load_ids = [&](int i0) {  // lane l: block l & 1 of this wavefront's step i0 + l / 2; only blocks that hold keys of the range are named
      const int blk = 2 * (s_first + wave + kWaves * (i0 + (lane >> 1))) + (lane & 1);
      return table[min(max(blk, blk_lo), blk_hi)];
    };
    int ids = 0, ids_next = 0;
    if (count > 0) {
      ids = load_ids(0);
      if (count > 32) ids_next = load_ids(32);
    }
    const char* const k_head = k_cache + (size_t)g * blk_bytes;
    const char* const v_head = v_cache + (size_t)g * blk_bytes;
    const uint8_t* const s_head = Frag::kNarrow ? scales + (size_t)g * kScaleBytes : nullptr;
    const int units = D / C::kUnit;
    int k_off[Frag::NK];  // (units behind the head vector: its first one, which meets zeros of Q)
#pragma unroll
    for (int j = 0; j < Frag::NK; ++j) {
      const int unit = 4 * j + quad;
      k_off[j] = (unit < units ? unit : 0) * 256 + ((8 * (col >> 2) + (col & 3)) & 15) * 16;
    }
    const int v_off = (col * kBlockSize + 8 * (quad & 1)) * C::kBytes;
    auto load = [&](Frag& f, int i) {
      if ((i & 31) == 0 && i > 0) {
        ids = ids_next;
        if (i + 32 < count) ids_next = load_ids(i + 32);
      }
      const int id0 = __builtin_amdgcn_readlane(ids, 2 * (i & 31)), id1 = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + 1);
      const long long at0 = (long long)id0 * blk_stride, at1 = (long long)id1 * blk_stride;
      const char* const kp = k_head + (col >= 8 ? at1 : at0);
      const char* const vp = v_head + (quad >= 2 ? at1 : at0) + v_off;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < Frag::NK; ++j) f.k[t][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + k_off[j] + 64 * t));
      if constexpr (Frag::kNarrow) {
        const uint8_t* const sp = s_head + (long long)(quad >= 2 ? id1 : id0) * Hkv * kScaleBytes + 8 * (quad & 1);
        f.sk = *reinterpret_cast<const u32x2*>(sp);
        f.sv = *reinterpret_cast<const u32x2*>(sp + kBlockSize);
      }
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt)
        if (16 * dt < D) f.v[dt] = __builtin_nontemporal_load(reinterpret_cast<const typename Frag::VReg*>(vp + dt * 16 * kBlockSize * C::kBytes));
    };

    // ---- a step
    f32x4 acc[2 * NC];
#pragma unroll
    for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kLowest, l = 0.f;
    auto process = [&](Frag& f, int i) {
      const int k0 = 32 * (s_first + wave + kWaves * i);
      f32x4 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          bf16x8 a;
          if constexpr (Frag::kNarrow) a = codes_to_bf16x8<F>(f.k[t][c >> 1][2 * (c & 1)], f.k[t][c >> 1][2 * (c & 1) + 1], 1.f);
          else a = __builtin_bit_cast(bf16x8, f.k[t][c]);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[c], s[t], 0, 0, 0);
        }
      }
      // Keys outside the range (stale slots, tokens that a window has passed): their scores are excluded and what stands in their place is
      // cleared, since 0 times a stale NaN would reach the sums.
      const bool edge = k0 < lo || k0 + 32 > hi;
      const int first = lo - k0 - 8 * quad, last = hi - k0 - 8 * quad;  // of the lane's 8 tokens: [first, last)
      if (edge) {
        u32x4 keep;  // halves of words: all bits of the tokens that stay
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t even_ok = 2 * w >= first && 2 * w < last, odd_ok = 2 * w + 1 >= first && 2 * w + 1 < last;
          keep[w] = (even_ok ? 0xffffu : 0u) | (odd_ok ? 0xffff0000u : 0u);
        }
        if constexpr (Frag::kNarrow) {
          const uint32_t a = __builtin_amdgcn_perm(keep[1], keep[0], 0x06040200u), c = __builtin_amdgcn_perm(keep[3], keep[2], 0x06040200u);
          f.sk[0] &= a, f.sk[1] &= c, f.sv[0] &= a, f.sv[1] &= c;
#pragma unroll
          for (int dt = 0; dt < 2 * NC; ++dt) f.v[dt][0] &= a, f.v[dt][1] &= c;
        } else {
#pragma unroll
          for (int dt = 0; dt < 2 * NC; ++dt)
#pragma unroll
            for (int w = 0; w < 4; ++w) f.v[dt][w] &= keep[w];
        }
      }
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = s[j >> 2][j & 3];
      if constexpr (Frag::kNarrow) {
        x[0] *= scale_of<0>(f.sk[0]), x[1] *= scale_of<1>(f.sk[0]), x[2] *= scale_of<2>(f.sk[0]), x[3] *= scale_of<3>(f.sk[0]);
        x[4] *= scale_of<0>(f.sk[1]), x[5] *= scale_of<1>(f.sk[1]), x[6] *= scale_of<2>(f.sk[1]), x[7] *= scale_of<3>(f.sk[1]);
      }
      if (kForm && cap_in > 0.f) {
        // cap tanh(y) = cap - 2 cap / (1 + exp(2 y)), off by an ulp of the cap
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = cap_log2e - 2.f * cap_log2e * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[j] * cap_in));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= scale_log2e;
      }
      if (kForm && slopes) {
        const int away = k0 + 8 * quad - position;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(slope, (float)(away + j), x[j]);
      }
      if (edge) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < first || j >= last) x[j] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = across_quads_max(top);
      if (__any(top - m > kTau)) {
        const float m_new = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - m_new);
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] *= alpha;
        m = m_new;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(x[j] - m);
      l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      if constexpr (Frag::kNarrow) {
        x[0] *= scale_of<0>(f.sv[0]), x[1] *= scale_of<1>(f.sv[0]), x[2] *= scale_of<2>(f.sv[0]), x[3] *= scale_of<3>(f.sv[0]);
        x[4] *= scale_of<0>(f.sv[1]), x[5] *= scale_of<1>(f.sv[1]), x[6] *= scale_of<2>(f.sv[1]), x[7] *= scale_of<3>(f.sv[1]);
      }
      const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])});
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt)
        if (16 * dt < D) {
          bf16x8 a;
          if constexpr (Frag::kNarrow) a = codes_to_bf16x8<F>(f.v[dt][0], f.v[dt][1], 1.f);
          else a = __builtin_bit_cast(bf16x8, f.v[dt]);
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p, acc[dt], 0, 0, 0);
        }
    };
    {
      Frag f0, f1;
      if (count > 0) load(f0, 0);
      for (int i = 0; i < count; i += 2) {
        if (i + 1 < count) load(f1, i + 1);
        process(f0, i);
        if (i + 1 >= count) break;
        if (i + 2 < count) load(f0, i + 2);
        process(f1, i + 1);
      }
    }

    // ---- the wavefronts' states, added up
    l = across_quads_sum(l);
    if (quad == 0) s_m[wave][col] = m, s_l[wave][col] = l;
    __syncthreads();
    {
      const float M = fmaxf(fmaxf(s_m[0][col], s_m[1][col]), fmaxf(s_m[2][col], s_m[3][col])), alpha = __builtin_amdgcn_exp2f(m - M);
#pragma unroll
      for (int dt = 0; dt < 2 * NC; ++dt) acc[dt] *= alpha;
      if (wave == 0 && quad == 0) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += s_l[w][col] * __builtin_amdgcn_exp2f(s_m[w][col] - M);
        s_M[col] = M;
        s_L[col] = sum;
      }
    }
    const int slot = (int)(from >> 16) + k_slice;
    float* const state = states + ((size_t)slot * Hkv + g) * G * state_words;  // (read for cut sequences alone)
    const __amdgpu_buffer_rsrc_t to_state = __builtin_amdgcn_make_buffer_rsrc(state, 0, G * state_words * 4, kRsrc);
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      if (pass > 0) __syncthreads();
      if (col < G)
#pragma unroll
        for (int dt = 0; dt < kCh / 16; ++dt)
          *reinterpret_cast<f32x4*>(s_o + ((size_t)wave * G + col) * kRow + 16 * dt + 4 * quad) = acc[pass * (kCh / 16) + dt];
      __syncthreads();
      for (int i = tid; i < G * (kCh / 4); i += kThreads) {
        const int h = i / (kCh / 4), at = 4 * (i % (kCh / 4)), d = pass * kCh + at;
        if (d >= D) continue;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o += *reinterpret_cast<const f32x4*>(s_o + ((size_t)w * G + h) * kRow + at);
        if (n_slices == 1) {
          const float inv = 1.f / s_L[h];
          *reinterpret_cast<u32x2*>(out_rows + (size_t)h * D + d) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        } else {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), to_state, (h * state_words + d) * 4, 0, kAgent);
        }
      }
    }
    if (n_slices == 1) {
      if (lse_rows && tid < G) lse_rows[tid] = (s_M[tid] + log2f(s_L[tid])) * kLn2;
      __syncthreads();
      continue;
    }
    if (tid < G)
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(s_M[tid]), __float_as_uint(s_L[tid])}, to_state, (tid * state_words + D) * 4, 0, kAgent);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_order = (int)atomicInc(counters + (size_t)b * Hkv + g, (unsigned)n_slices - 1);  // (the last one wraps it to zero)
    __syncthreads();
    if (s_order != n_slices - 1) continue;  // (s_order is written again behind two barriers at least)

    // ---- the last workgroup of the (sequence, head): all slices' states, in order
    const int between = Hkv * G * state_words;  // floats from slice to slice
    const __amdgpu_buffer_rsrc_t from_states = __builtin_amdgcn_make_buffer_rsrc(states + ((size_t)(from >> 16) * Hkv + g) * G * state_words, 0,
                                                                                 ((n_slices - 1) * between + G * state_words) * 4, kRsrc);
    float* const s_w = s_o;  // [G][n_slices]: weights of the slices
    for (int h = wave; h < G; h += kWaves) {
      constexpr int kMost = kScoredMostSlices / 64;
      float ms[kMost], ls[kMost], M = kLowest, L = 0.f;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        ms[i] = kLowest, ls[i] = 0.f;
        if (const int k = 64 * i + lane; k < n_slices) {
          const u32x2 ml = __builtin_amdgcn_raw_buffer_load_b64(from_states, (k * between + h * state_words + D) * 4, 0, kAgent);
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
        if (const int k = 64 * i + lane; k < n_slices) s_w[h * n_slices + k] = w;
      }
      L = wave_sum(L);
      if (lane == 0) s_M[h] = M, s_L[h] = L;
    }
    __syncthreads();
    // (parts of the slices, each of as many threads as the result has groups of four channels)
    const int groups = G * D / 4, parts = max(1, kThreads / groups);
    for (int base = 0; base < groups; base += kThreads) {
      const int part = parts > 1 ? tid / groups : 0, i = parts > 1 ? tid - part * groups : base + tid;
      const bool here = part < parts && i < groups;
      const int h = here ? i / (D / 4) : 0, d = here ? 4 * (i - h * (D / 4)) : 0;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      if (here) {
        constexpr int kAtOnce = 8;
        for (int k0 = part; k0 < n_slices; k0 += kAtOnce * parts) {
          f32x4 x[kAtOnce];
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j)  // (behind the last slice: that one again, not added)
            x[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_states, (min(k0 + j * parts, n_slices - 1) * between + h * state_words + d) * 4, 0, kAgent));
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j)
            if (k0 + j * parts < n_slices) o += x[j] * s_w[h * n_slices + k0 + j * parts];
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
    __syncthreads();
  }
}

template <int F, int NC>
void launch_formed(const ScoredArgs& a, hipStream_t s) {
  const int G = a.Hq / a.Hkv;
  const bool form = a.softcap > 0.f || a.slopes;
  // states of four wavefronts, or the weights of the slices when they are added up
  const size_t words = std::max((size_t)kWaves * G * (kPassChannels<NC> + 4), (size_t)G * kScoredMostSlices);
  const size_t lds = (head_words(a.B) + words) * sizeof(uint32_t);
  const float cap_in = form && a.softcap > 0.f ? 2.f * a.scale_log2e / a.softcap : 0.f;
  const int64_t most = (int64_t)a.B * a.Hkv + decode_scored_slices(a.num_cu);  // items there can be
  const int grid = (int)std::min<int64_t>(decode_scored_grid(a.num_cu), most);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), lds, s, (const uint16_t*)a.q, a.q_row_stride, (const char*)a.k_cache, (const char*)a.v_cache, a.scales,
                       a.block_table, a.bt_stride, a.ctx_before, a.key_begin, a.key_end, a.slopes, (uint16_t*)a.out, a.lse, a.states, a.counters, a.B, a.Hq, a.Hkv, G,
                       a.D, decode_scored_slices(a.num_cu), a.scale_log2e, cap_in, a.softcap * kLog2e);
  };
  if (form) go(&decode_scored_kernel<F, NC, true>);
  else go(&decode_scored_kernel<F, NC, false>);
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
