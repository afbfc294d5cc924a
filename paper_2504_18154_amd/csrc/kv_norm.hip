// KV-cache append with each head of K and Q normed and turned, and K and V coded, on the way; and the cached rows read back.
//
// A row (token, head) is D elements, 8 to a lane: 8, 16 or 32 lanes of a wavefront hold it (D <= 64, 128, 256), sum its squares and find its largest magnitude
// among themselves.  All of it is fp32, rounded once: to bf16, or to codes (quant.h).
//   norm      y = x / sqrt(mean(x^2) + eps) * w
//   rotation  pair (a, b) -> (a cos - b sin, a sin + b cos); kv_rope.hip says how the angles are formed.  A token's weights and angles make one pair of factors per
//             element, for itself and its partner.  Partners come from the lane that has them; where they are not
//             eight in a lane (rotary widths that are odd multiples of 8), from memory.
//   codes     the scale from the largest magnitude of the turned row, then one rounding
//
// Memory bounds the large calls, launch latency and a few round trips the small ones.  A lane keeps its token's factors and walks the heads, the next ones' loads
// in flight.  The blocks of the batch are numbered as in kv_append.hip; a workgroup takes the tokens of one block and a run of heads of K and Q, or up to four
// heads of V, whose codes go through LDS to lie along the slots.
// Measured, 64 query heads and 8 of K and V, of 128, rotated and normed: 65 536 tokens into 8-bit codes 506 us (2.55 GB, 5.0 TB/s, what a copy reaches), into bf16 600
// (4.5 TB/s: the 16 bytes that a lane has of a row of K go to a line of their own), three chunks of 200 ... 1500 tokens into bf16 38 us, a token of each of 64 sequences (40 query heads) 5.6 us.
#include <type_traits>

#include "quant.h"
#include "scored.h"
#include "turns.h"

namespace eco {

namespace {

constexpr int kThreads = 256;
constexpr int kVHeads = 4;  // heads of V to a workgroup
// Heads of K and Q to a workgroup from which its lanes work on two rows at a time.  72 heads of 65 536 tokens into codes: 573 us with one, 506 with two; into bf16 600 and
// 704.  7 heads of 2400 tokens: 38 with one, 47 with two, whose registers (116 for 86) leave fewer workgroups to a CU.
constexpr int kManyHeads = 16;
constexpr float kLeastEps = 0x1p-100f;  // of a norm, beside which squares below 2^-126 do not count

// Sum and maximum over the LP lanes that hold a row; every lane has the result, in the same order of sums everywhere.
template <int LP, typename Op>
__device__ __forceinline__ float over_row(float x, Op op) {
  auto moved = [&](auto ctrl) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
  x = op(x, moved(std::integral_constant<int, 0xb1>()));   // quad_perm: neighbours
  x = op(x, moved(std::integral_constant<int, 0x4e>()));   // quad_perm: pairs
  x = op(x, moved(std::integral_constant<int, 0x141>()));  // row_half_mirror: quads
  if (LP >= 16) x = op(x, moved(std::integral_constant<int, 0x140>()));  // row_mirror: halves of 16
  if (LP >= 32) x = op(x, __shfl_xor(x, 16));
  return x;
}

struct alignas(16) Eight {
  uint16_t e[8];
};
struct alignas(8) Four {
  uint16_t e[4];
};

struct NormArgs {
  const uint16_t *q, *k_new, *v_new;
  uint16_t* q_out;
  char *k_cache, *v_cache;
  uint8_t* scales;
  const float *q_weight, *k_weight;
  const int32_t *cu_q, *ctx_before, *block_table;
  int q_row_stride, q_out_row_stride, new_row_stride, bt_stride, B, Hq, Hkv, D, weight_stride;
  float eps, per_D;  // per_D: 1 / D, or 0 without a norm
};

// What a lane needs of its 8 elements' places: element i becomes x c[i] + (its partner) s[i].
template <bool kAdjacent>
struct Place {
  int e0, D;           // first element; lanes behind the row hold zeros
  bool here, turned;   // turned: all 8 are (rotary is a multiple of 8)
  bool exchanged;      // the partners are one lane's 8 elements (rotary is a multiple of 16)
  int from;            // that lane, for the exchange
  int away[2];         // else: of the partners of elements 0 .. 3 and 4 .. 7
  float c[8], s[8];
  __device__ __forceinline__ Place(int l, int D_) : e0(8 * l), D(D_), here(8 * l < D_), turned(false), exchanged(true), from(0) { away[0] = away[1] = 0; }
  __device__ __forceinline__ void angles(const Turns& turns, int tok, int position) {
    const int R = turns.rotary, half = R >> 1;
    turned = e0 < R;
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = 1.f, s[i] = -0.f;  // (a partner of 0 leaves x as it is, the sign of a zero too)
    exchanged = !(half & 7);
    from = 4 * ((int)(threadIdx.x & 63) + (e0 < half ? half : -half) / 8);
    if (!turned) return;
    if constexpr (kAdjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Angle t = angle_of_pair(turns, (e0 >> 1) + i, tok, position);
        c[2 * i] = c[2 * i + 1] = t.c;
        s[2 * i] = -t.s, s[2 * i + 1] = t.s;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool second = e0 + 4 * h >= half;
        away[h] = second ? -half : half;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Angle t = angle_of_pair(turns, e0 + 4 * h + i - (second ? half : 0), tok, position);
          c[4 * h + i] = t.c;
          s[4 * h + i] = second ? t.s : -t.s;
        }
      }
    }
  }
};

// A row's elements as they come, and their partners' where these have to be loaded.
template <bool kAdjacent>
struct Raw {
  u32x4 own, partner;
  __device__ __forceinline__ void load(const uint16_t* row, const Place<kAdjacent>& at) {
    partner = u32x4{0, 0, 0, 0};
    own = *reinterpret_cast<const u32x4*>(row + (at.here ? at.e0 : 0));
    if (!kAdjacent && !at.exchanged && at.turned)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(row + at.e0 + 4 * h + at.away[h]);
        partner[2 * h] = x[0], partner[2 * h + 1] = x[1];
      }
  }
  __device__ __forceinline__ void exchange(const Place<kAdjacent>& at) {
    if constexpr (kAdjacent) {
#pragma unroll
      for (int i = 0; i < 4; ++i) partner[i] = at.turned ? __builtin_amdgcn_alignbit(own[i], own[i], 16) : 0u;
    } else if (at.exchanged) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = (uint32_t)__builtin_amdgcn_ds_bpermute(at.from, (int)own[i]);
        partner[i] = at.turned ? x : 0u;
      }
    }
  }
};
// The factors of a row's elements and of their partners: the rotation's, times the weights (NULL: 1).
template <bool kAdjacent>
struct Factors {
  float own[8], partner[8];
  __device__ __forceinline__ void set(const float* w, const Place<kAdjacent>& at) {
#pragma unroll
    for (int i = 0; i < 8; ++i) own[i] = at.c[i], partner[i] = at.s[i];
    if (!w || !at.here) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(w + at.e0 + 4 * h);
      f32x4 b = a;
      if (kAdjacent) b = f32x4{a[1], a[0], a[3], a[2]};
      else if (at.turned) b = *reinterpret_cast<const f32x4*>(w + at.e0 + 4 * h + at.away[h]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        own[4 * h + i] *= a[i];
        if (at.turned) partner[4 * h + i] *= b[i];
      }
    }
  }
};
__device__ __forceinline__ void values_of(float (&y)[8], u32x4 x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
}

// per_D: 1 / D, or 0 without a norm
template <int LP, bool kAdjacent>
__device__ __forceinline__ void formed(float (&y)[8], Raw<kAdjacent>& raw, const Factors<kAdjacent>& by, const Place<kAdjacent>& at, float per_D, float eps) {
  float x[8], other[8];
  if (!at.here) raw.own = u32x4{0, 0, 0, 0};
  raw.exchange(at);
  values_of(x, raw.own);
  values_of(other, raw.partner);
  if (per_D > 0.f) {
    auto squares = [&]() {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
      return over_row<LP>(sum, [](float a, float b) { return a + b; });
    };
    float sum = squares();
    if (eps < kLeastEps) {  // (squares that fp32 has no bits for are the whole of the mean: they are taken of the row times 2^80)
      const bool tiny = sum < 0x1p-60f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tiny ? x[i] * 0x1p80f : x[i], other[i] = tiny ? other[i] * 0x1p80f : other[i];
      sum = squares();
      eps = tiny ? eps * 0x1p80f * 0x1p80f : eps;
    }
    const float f = rsqrtf(__builtin_fmaf(sum, per_D, eps));
    // (before the weights and the rotation: what is large stays inside fp32)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= f, other[i] *= f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(other[i], by.partner[i], x[i] * by.own[i]);
}

// Codes of a row's 8 elements, and its scale byte.
template <int LP, int F>
__device__ __forceinline__ u32x2 coded(const float (&y)[8], uint32_t& byte) {
  // (the largest magnitude by its bits, so that a NaN is the largest)
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(y[i]) & 0x7fffffffu);
  most = __float_as_uint(over_row<LP>(__uint_as_float(most), [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
  byte = scale_byte<F>(__uint_as_float(most));
  if (byte == kBadScale) return u32x2{0, 0};
  const float f = inverse_scale(byte);
  return u32x2{to_codes<F>(y[0] * f, y[1] * f, y[2] * f, y[3] * f), to_codes<F>(y[4] * f, y[5] * f, y[6] * f, y[7] * f)};
}
__device__ __forceinline__ Eight rounded8(const float (&y)[8]) {
  return __builtin_bit_cast(Eight, u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])});
}

// A K row into its block of one head, or a Q row out.
template <int LP, int F>
__device__ __forceinline__ void store_k(char* head, uint8_t* scale, int slot, int l, bool here, const float (&y)[8]) {
  if constexpr (F == kNative) {
    if (here) *reinterpret_cast<Eight*>(head + l * 256 + slot * 16) = rounded8(y);
  } else {
    uint32_t byte;
    const u32x2 c = coded<LP, F>(y, byte);
    if (here) *reinterpret_cast<u32x2*>(head + (l >> 1) * 256 + slot * 16 + (l & 1) * 8) = c;
    if (l == 0) scale[slot] = (uint8_t)byte;
  }
}

__device__ __forceinline__ void transpose4(const uint32_t (&r)[4], uint32_t (&o)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(c, a, 0x05040100u), o[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(d, b, 0x05040100u), o[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// kAhead: rows of a lane that are loaded while as many are worked on.
template <int LP, int F, bool kAdjacent, int kAhead>
__global__ __launch_bounds__(kThreads) void kv_append_norm_kernel(const NormArgs a, const Turns turns, int v_slices, int per_slice) {
  constexpr int kBytes = Cached<F>::kBytes, kGroups = kThreads / LP;
  extern __shared__ __attribute__((aligned(16))) char staged[];
  const int D = a.D, Hkv = a.Hkv, tid = threadIdx.x, group = tid / LP, l = tid % LP;
  auto first_unit = [](int cu, int b) { return (cu >> 4) + 2 * b; };
  const SeqOf seq = find_sequence(a.cu_q, a.ctx_before, a.B, blockIdx.x, first_unit);
  const int b = seq.b, tok0 = seq.tok0, S = seq.S, cb = seq.cb, nth = (int)blockIdx.x - first_unit(tok0, b);
  if (S <= 0 || nth > ((cb + S - 1) >> 4) - (cb >> 4)) return;
  const int j = (cb >> 4) + nth;
  if (j < 0) return;  // (tokens at negative positions: places of a padded batch)
  const int lo = max(0, cb - (j << 4)), hi = min(16, cb + S - (j << 4));  // addressed slots of the block
  const int t_slot0 = tok0 + (j << 4) - cb;                               // packed token of slot 0 (may lie before tok0)
  const size_t blk = (size_t)a.block_table[(size_t)b * a.bt_stride + j];
  const size_t head_bytes = (size_t)kBlockSize * D * kBytes;

  if ((int)blockIdx.y < v_slices) {
    const int g0 = blockIdx.y * kVHeads, heads = min(kVHeads, Hkv - g0);
    char* const dst = a.v_cache + (blk * Hkv + g0) * head_bytes;
    constexpr int kRows = kVHeads * 16 / kGroups;
    u32x4 x[kRows];
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
      // (rows and lanes that there are not: others' places, so that no load waits for a branch)
      const int r = group + n * kGroups, slot = min(max(r & 15, lo), hi - 1), h = min(r >> 4, heads - 1);
      x[n] = *reinterpret_cast<const u32x4*>(a.v_new + (size_t)(t_slot0 + slot) * a.new_row_stride + (size_t)(g0 + h) * D + (8 * l < D ? 8 * l : 0));
    }
    if constexpr (F != kNative) {
      const int row_bytes = D + 8;
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        const int r = group + n * kGroups, slot = r & 15;
        if (r >= heads * 16 || slot < lo || slot >= hi) continue;
        float y[8];
        values_of(y, 8 * l < D ? x[n] : u32x4{0, 0, 0, 0});
        uint32_t byte;
        const u32x2 c = coded<LP, F>(y, byte);
        if (8 * l < D) *reinterpret_cast<u32x2*>(staged + r * row_bytes + 8 * l) = c;
        if (l == 0) a.scales[(blk * Hkv + g0 + (r >> 4)) * kScaleBytes + kBlockSize + slot] = (uint8_t)byte;
      }
      __syncthreads();
      for (int u = tid; u < heads * (D / 4); u += kThreads) {
        const int h = u / (D / 4), d = 4 * (u - h * (D / 4));
        uint32_t w[4][4];  // [channel][four slots]
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          uint32_t r[4], o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = *reinterpret_cast<const uint32_t*>(staged + (h * 16 + 4 * s + i) * row_bytes + d);
          transpose4(r, o);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i][s] = o[i];
        }
        char* const to = dst + h * head_bytes + d * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (lo == 0 && hi == 16) {
            *reinterpret_cast<u32x4*>(to + i * 16) = u32x4{w[i][0], w[i][1], w[i][2], w[i][3]};
          } else {
#pragma unroll
            for (int s = 0; s < 16; ++s)
              if (s >= lo && s < hi) to[i * 16 + s] = (char)(w[i][s >> 2] >> (8 * (s & 3)));
          }
        }
      }
    } else {
      const int vrow = D + 8;
      uint16_t* const vt = reinterpret_cast<uint16_t*>(staged);
#pragma unroll
      for (int n = 0; n < kRows; ++n)
        if (const int r = group + n * kGroups; r < heads * 16 && 8 * l < D) *reinterpret_cast<u32x4*>(vt + r * vrow + 8 * l) = x[n];
      __syncthreads();
      // two channels' halves of the slots to a thread
      for (int u = tid; u < heads * D; u += kThreads) {
        const int s0 = 8 * (u & 1), h = (u >> 1) / (D / 2), d = 2 * ((u >> 1) - h * (D / 2));
        const uint16_t* const from = vt + (h * 16 + s0) * vrow + d;
        uint16_t* const to = reinterpret_cast<uint16_t*>(dst) + ((size_t)h * D + d) * 16 + s0;
        u32x4 y[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t even = *reinterpret_cast<const uint32_t*>(from + 2 * w * vrow), odd = *reinterpret_cast<const uint32_t*>(from + (2 * w + 1) * vrow);
          y[0][w] = __builtin_amdgcn_perm(odd, even, 0x05040100u);
          y[1][w] = __builtin_amdgcn_perm(odd, even, 0x07060302u);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (s0 >= lo && s0 + 8 <= hi) {
            *reinterpret_cast<u32x4*>(to + i * 16) = y[i];
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (s0 + e >= lo && s0 + e < hi) to[i * 16 + e] = (uint16_t)(y[i][e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    }
    return;
  }

  // K heads, then Q heads: h_begin .. h_end - 1 of the list
  const int total = Hkv + (a.q ? a.Hq : 0), h_begin = ((int)blockIdx.y - v_slices) * per_slice, h_end = min(h_begin + per_slice, total);
  constexpr int kSlots = kGroups < 16 ? kGroups : 16, kHeads = kGroups / kSlots;  // that the workgroup has at a time
  for (int slot = group % kSlots; slot < 16; slot += kSlots) {
    if (slot < lo || slot >= hi) continue;
    const int tok = t_slot0 + slot;
    Place<kAdjacent> at(l, D);
    at.angles(turns, tok, (j << 4) + slot);
    Factors<kAdjacent> by;
    int by_of = -1;  // 0: K's, 1: Q's
    const int step = kAhead * kHeads;
    Raw<kAdjacent> next[kAhead];
    auto load = [&](int h0) {
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = min(h0 + n * kHeads, h_end - 1);
        next[n].load(h < Hkv ? a.k_new + (size_t)tok * a.new_row_stride + (size_t)h * D : a.q + (size_t)tok * a.q_row_stride + (size_t)(h - Hkv) * D, at);
      }
    };
    int h0 = h_begin + group / kSlots;
    load(h0);
    for (; h0 < h_end; h0 += step) {
      Raw<kAdjacent> raw[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) raw[n] = next[n];
      if (h0 + step < h_end) load(h0 + step);
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = h0 + n * kHeads;
        if (h >= h_end) break;
        const bool is_q = h >= Hkv;
        if (by_of != (int)is_q || a.weight_stride) {
          const float* const base = is_q ? a.q_weight : a.k_weight;
          by.set(base ? base + (size_t)(is_q ? h - Hkv : h) * a.weight_stride : nullptr, at);
          by_of = is_q;
        }
        float y[8];
        formed<LP>(y, raw[n], by, at, a.per_D, a.eps);
        if (is_q) {
          if (at.here) *reinterpret_cast<Eight*>(a.q_out + (size_t)tok * a.q_out_row_stride + (size_t)(h - Hkv) * D + 8 * l) = rounded8(y);
        } else {
          store_k<LP, F>(a.k_cache + (blk * Hkv + h) * head_bytes, a.scales + (blk * Hkv + h) * kScaleBytes, slot, l, at.here, y);
        }
      }
    }
  }
}

// At most one new token per sequence (the decode step): a row of K, of V or of Q to a group of lanes, each with its own angles and weights.
template <int LP, int F, bool kAdjacent>
__global__ __launch_bounds__(kThreads) void kv_append_norm_one_kernel(const NormArgs a, const Turns turns, int rows_of_seq) {
  constexpr int kBytes = Cached<F>::kBytes;
  const int D = a.D, Hkv = a.Hkv, l = threadIdx.x % LP;
  const long long row = (long long)blockIdx.x * (blockDim.x / LP) + threadIdx.x / LP;
  const int b = (int)(row / rows_of_seq), r = (int)(row - (long long)b * rows_of_seq);
  if (b >= a.B) return;
  const int p = a.ctx_before[b], tok = a.cu_q[b];
  if (a.cu_q[b + 1] - tok <= 0 || p < 0) return;
  const int slot = p & 15;
  const bool is_k = r < Hkv, is_q = r >= 2 * Hkv;
  const int h = is_q ? r - 2 * Hkv : is_k ? r : r - Hkv;
  const size_t blk = is_q ? 0 : (size_t)a.block_table[(size_t)b * a.bt_stride + (p >> 4)], head_bytes = (size_t)kBlockSize * D * kBytes;
  if (!is_k && !is_q) {
    Eight x = {};
    if (8 * l < D) x = *reinterpret_cast<const Eight*>(a.v_new + (size_t)tok * a.new_row_stride + (size_t)h * D + 8 * l);
    char* const to = a.v_cache + (blk * Hkv + h) * head_bytes;
    if constexpr (F == kNative) {
      if (8 * l < D)
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(to)[(8 * l + i) * 16 + slot] = x.e[i];
    } else {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = bf16_bits_to_float(x.e[i]);
      uint32_t byte;
      const u32x2 c = coded<LP, F>(y, byte);
      if (8 * l < D)
#pragma unroll
        for (int i = 0; i < 8; ++i) to[(8 * l + i) * 16 + slot] = (char)(c[i >> 2] >> (8 * (i & 3)));
      if (l == 0) a.scales[(blk * Hkv + h) * kScaleBytes + kBlockSize + slot] = (uint8_t)byte;
    }
    return;
  }
  Place<kAdjacent> at(l, D);
  const uint16_t* const src = is_q ? a.q + (size_t)tok * a.q_row_stride + (size_t)h * D : a.k_new + (size_t)tok * a.new_row_stride + (size_t)h * D;
  at.angles(turns, tok, p);
  Raw<kAdjacent> raw;
  raw.load(src, at);
  Factors<kAdjacent> by;
  const float* const base = is_q ? a.q_weight : a.k_weight;
  by.set(base ? base + (size_t)h * a.weight_stride : nullptr, at);
  float y[8];
  formed<LP>(y, raw, by, at, a.per_D, a.eps);
  if (is_q) {
    if (at.here) *reinterpret_cast<Eight*>(a.q_out + (size_t)tok * a.q_out_row_stride + (size_t)h * D + 8 * l) = rounded8(y);
  } else {
    store_k<LP, F>(a.k_cache + (blk * Hkv + h) * head_bytes, a.scales + (blk * Hkv + h) * kScaleBytes, slot, l, at.here, y);
  }
}

template <int LP, int F, bool kAdjacent>
void launch_append(const NormAppend& a, const NormArgs& args, const Turns& turns, hipStream_t s) {
  if (a.max_new_len <= 1) {
    const int of_seq = 2 * a.Hkv + (a.q ? a.Hq : 0);
    const int64_t rows = (int64_t)a.B * of_seq, waves = (rows * LP + 63) / 64;
    const int threads = waves <= 2 * a.num_cu ? 64 : kThreads, at_once = threads / LP;
    hipLaunchKernelGGL((kv_append_norm_one_kernel<LP, F, kAdjacent>), dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(threads), 0, s, args, turns, of_seq);
    return;
  }
  const int v_slices = (a.Hkv + kVHeads - 1) / kVHeads, total = a.Hkv + (a.q ? a.Hq : 0);
  const int64_t units = (int64_t)a.T / 16 + 2 * (int64_t)a.B;
  // heads per workgroup: eight workgroups per CU, then more heads to an angle
  const int64_t want = (8 * (int64_t)a.num_cu + units - 1) / units;
  const int slices = (int)(want < total ? want : total), per_slice = (total + slices - 1) / slices;
  const dim3 grid((unsigned)units, (unsigned)(v_slices + (total + per_slice - 1) / per_slice));
  const size_t lds = (size_t)kVHeads * 16 * (F == kNative ? 2 * (a.D + 8) : a.D + 8);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, s, args, turns, v_slices, per_slice); };
  if (F != kNative && per_slice >= kManyHeads) go(&kv_append_norm_kernel<LP, F, kAdjacent, 2>);
  else go(&kv_append_norm_kernel<LP, F, kAdjacent, 1>);
}

// Workgroup x: a block of a sequence, numbered as above; y: up to `heads_of` heads.
template <int F>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const char* __restrict__ k_cache, const char* __restrict__ v_cache, const uint8_t* __restrict__ scales,
                                                           uint16_t* __restrict__ k_rows, uint16_t* __restrict__ v_rows, int row_stride, const int32_t* __restrict__ cu,
                                                           const int32_t* __restrict__ first, const int32_t* __restrict__ block_table, int bt_stride, int B, int Hkv, int D,
                                                           int heads_of) {
  typedef Cached<F> C;
  constexpr int kUnit = C::kUnit;
  extern __shared__ __attribute__((aligned(16))) char staged[];
  auto first_unit = [](int c, int b) { return (c >> 4) + 2 * b; };
  const SeqOf seq = find_sequence(cu, first, B, blockIdx.x, first_unit);
  const int nth = (int)blockIdx.x - first_unit(seq.tok0, seq.b);
  if (seq.S <= 0 || nth > ((seq.cb + seq.S - 1) >> 4) - (seq.cb >> 4)) return;
  const int j = (seq.cb >> 4) + nth, tid = threadIdx.x;
  if (j < 0) return;
  const int lo = max(0, seq.cb - (j << 4)), hi = min(16, seq.cb + seq.S - (j << 4)), t_slot0 = seq.tok0 + (j << 4) - seq.cb;
  const size_t blk = (size_t)block_table[(size_t)seq.b * bt_stride + j], head_bytes = (size_t)kBlockSize * D * C::kBytes;
  const int g0 = blockIdx.y * heads_of, heads = min(heads_of, Hkv - g0);
  const uint8_t* const sc = F == kNative ? nullptr : scales + (blk * Hkv + g0) * kScaleBytes;
  auto scale = [&](uint32_t byte) { return byte == kBadScale ? NAN : scale_of_byte(byte); };

  if (k_rows) {
    const char* const src = k_cache + (blk * Hkv + g0) * head_bytes;
    const int units = D / kUnit;
    for (int u = tid; u < heads * units * 16; u += kThreads) {
      const int slot = u & 15, hu = u >> 4, h = hu / units, c = hu - h * units;
      if (slot < lo || slot >= hi) continue;
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + (size_t)u * 16);
      uint16_t* const to = k_rows + (size_t)(t_slot0 + slot) * row_stride + (size_t)(g0 + h) * D + c * kUnit;
      if constexpr (F == kNative) {
        *reinterpret_cast<u32x4*>(to) = x;
      } else {
        const float f = scale(sc[h * kScaleBytes + slot]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y[8];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t v = x[2 * i + w];
            y[4 * w] = code_value<F, 0>(v) * f, y[4 * w + 1] = code_value<F, 1>(v) * f, y[4 * w + 2] = code_value<F, 2>(v) * f, y[4 * w + 3] = code_value<F, 3>(v) * f;
          }
          reinterpret_cast<Eight*>(to)[i] = rounded8(y);
        }
      }
    }
  }
  if (!v_rows) return;
  // V lies along the slots: 16 bytes at a time into LDS as they are, out as rows
  const char* const src = v_cache + (blk * Hkv + g0) * head_bytes;
  constexpr int kPitch = kBlockSize * C::kBytes + 4;  // of a channel in LDS
  for (int u = tid; u < heads * D * C::kBytes; u += kThreads) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(src + (size_t)u * 16);
    uint32_t* const to = reinterpret_cast<uint32_t*>(staged + (u / C::kBytes) * kPitch + (u % C::kBytes) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = x[i];
  }
  __syncthreads();
  for (int u = tid; u < heads * 16 * (D / 8); u += kThreads) {
    const int c = u % (D / 8), r = u / (D / 8), slot = r & 15, h = r >> 4;
    if (slot < lo || slot >= hi) continue;
    const char* const from = staged + (h * D + 8 * c) * kPitch + slot * C::kBytes;
    uint16_t* const to = v_rows + (size_t)(t_slot0 + slot) * row_stride + (size_t)(g0 + h) * D + 8 * c;
    if constexpr (F == kNative) {
      Eight x;
#pragma unroll
      for (int i = 0; i < 8; ++i) x.e[i] = *reinterpret_cast<const uint16_t*>(from + i * kPitch);
      *reinterpret_cast<Eight*>(to) = x;
    } else {
      const float f = scale(sc[h * kScaleBytes + kBlockSize + slot]);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = code_value<F, 0>(*reinterpret_cast<const uint8_t*>(from + i * kPitch)) * f;
      *reinterpret_cast<Eight*>(to) = rounded8(y);
    }
  }
}

}  // namespace

hipError_t launch_kv_append_norm(const NormAppend& a, const ecoserve_rope* rope, const double* inv_freq, const int32_t* positions, hipStream_t s) {
  Turns turns = {};
  if (rope) turns = make_turns(*rope, inv_freq, positions, a.T);
  const bool adjacent = rope && rope->pairing == ECOSERVE_ROPE_ADJACENT;
  const NormArgs args = {(const uint16_t*)a.q, (const uint16_t*)a.k_new, (const uint16_t*)a.v_new, (uint16_t*)a.q_out, (char*)a.k_cache, (char*)a.v_cache, a.scales,
                         a.norm ? a.q_weight : nullptr, a.norm ? a.k_weight : nullptr, a.cu_q, a.ctx_before, a.block_table, a.q_row_stride, a.q_out_row_stride, a.new_row_stride, a.bt_stride, a.B, a.Hq, a.Hkv,
                         a.D, a.norm ? a.weight_stride : 0, a.eps, a.norm ? 1.f / (float)a.D : 0.f};
  auto with_lanes = [&](auto format, auto pairing) {
    constexpr int F = decltype(format)::value;
    constexpr bool kAdjacent = decltype(pairing)::value;
    if (a.D <= 64) launch_append<8, F, kAdjacent>(a, args, turns, s);
    else if (a.D <= 128) launch_append<16, F, kAdjacent>(a, args, turns, s);
    else launch_append<32, F, kAdjacent>(a, args, turns, s);
  };
  auto with_format = [&](auto format) { adjacent ? with_lanes(format, std::true_type()) : with_lanes(format, std::false_type()); };
  switch (a.format) {
    case kInt8: with_format(std::integral_constant<int, kInt8>()); break;
    case kE4m3: with_format(std::integral_constant<int, kE4m3>()); break;
    default: with_format(std::integral_constant<int, kNative>()); break;
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const ReadBack& a, hipStream_t s) {
  const int64_t units = (int64_t)a.T / 16 + 2 * (int64_t)a.B;
  const int heads_of = units * a.Hkv <= 8 * (int64_t)a.num_cu ? 1 : a.D <= 128 ? 4 : 2;
  const dim3 grid((unsigned)units, (unsigned)((a.Hkv + heads_of - 1) / heads_of));
  auto go = [&](auto format) {
    constexpr int F = decltype(format)::value;
    const size_t lds = (size_t)heads_of * a.D * (kBlockSize * Cached<F>::kBytes + 4);
    hipLaunchKernelGGL(kv_read_kernel<F>, grid, dim3(kThreads), lds, s, (const char*)a.k_cache, (const char*)a.v_cache, a.scales, (uint16_t*)a.k_rows, (uint16_t*)a.v_rows,
                       a.row_stride, a.cu, a.first, a.block_table, a.bt_stride, a.B, a.Hkv, a.D, heads_of);
  };
  switch (a.format) {
    case kInt8: go(std::integral_constant<int, kInt8>()); break;
    case kE4m3: go(std::integral_constant<int, kE4m3>()); break;
    default: go(std::integral_constant<int, kNative>()); break;
  }
  return hipGetLastError();
}

}  // namespace eco
