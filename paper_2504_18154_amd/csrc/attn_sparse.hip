// Attention over listed blocks of the paged cache (Eq. 2 of Section 2.1 over the keys of the blocks in a list), for decode
// steps and prompts alike: every (token, K/V head) has a list of its own.
//
// The unit of work is one (token, K/V head): its G query heads are the columns of the products.
//   scores  S^T[key][head] = K . Q^T      values  O^T[d][head] += V^T . P^T
// bf16: two blocks at a time, 32 keys, v_mfma_f32_16x16x32_bf16 throughout.  The rows of the two score products are keys 8 q + i and 8 q + 4 + i (q the row
// of lanes, i < 4), so that a lane's eight weights are the eight keys that the second product's operand wants of it.  The weights go in two bf16 parts (16
// bits); the first is the weight less 1/128 of it, so that the second is never zero: an infinite value meets two weights that are not.  K comes in
// operand layout.  V's operand, eight keys of a channel, is not what lanes in a row find in a row in memory (64 requests an instruction, of 8
// bytes each); so it is asked for 1 KiB in a row and turned over in LDS.
// fp32: block by block, v_mfma_f32_16x16x4_f32, both in operand layout.
// Many tokens of bf16 prompts share what their lists have in common: attn_sparse_prompt_kernel, below.
//
// A workgroup of four wavefronts has one list, or a part of it where there are few; the wavefronts take its entries in turn, with the
// next blocks on their way (entries without keys are dropped before any load).  Their states are added up through LDS, those of parts by the workgroup
// that is done last with the list.  Bound by reading K and V: from memory in a decode step, from the caches behind prompts, whose neighbouring tokens list
// much the same blocks; the K/V heads go to different XCDs (consecutive workgroups), so that an XCD's cache holds the blocks of one or a few.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "sparse.h"

namespace eco {

namespace {

constexpr int kWaves = 4;
constexpr int kRsrc = 0x00020000;  // buffer descriptor: untyped 32-bit data, no swizzle, no stride
constexpr int kAgent = 16;         // past the caches that XCDs do not share
typedef const void __attribute__((address_space(1)))* gptr_t;
typedef void __attribute__((address_space(3)))* lptr_t;
constexpr float kRaise = 8.f;      // the exponent offset is raised when a score exceeds it by more (log2 units; 2^8: 256, below)
constexpr float kLowest = -3.402823466e38f;  // the offset of keys that all score -inf: their weights are 0, and there are keys

// The state of 16 columns: m exponent offset (-inf: no key yet, kLowest or more: keys), l this lane's share of the sum, o unnormalised.
template <int NV>
struct State {
  float m = -INFINITY, l = 0.f;
  f32x4 o[NV];
  // the offset follows the largest score (of this lane: top) of the columns
  __device__ __forceinline__ void raise(float top) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float raised = top > m + kRaise ? top : m, by = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - raised);
    l *= by;
#pragma unroll
    for (int dt = 0; dt < NV; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[dt][i] *= by;
    m = raised;
  }
  template <int N>
  static __device__ __forceinline__ float largest(const f32x4 (&s)[N]) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < N; ++t) top = fmaxf(top, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
    return top;
  }
  // scores q.k to weights; -inf: no key, or one that scores so (every column has a key: m is above -inf from here on)
  template <int N>
  __device__ __forceinline__ void weights(f32x4 (&s)[N], float scale_log2e) {
    const float top = fmaxf(largest(s) * scale_log2e, kLowest);
    if (__any(top > m + kRaise)) raise(top);
#pragma unroll
    for (int t = 0; t < N; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale_log2e, -m));
      l += (s[t][0] + s[t][1]) + (s[t][2] + s[t][3]);
    }
  }
  // The same of 32 keys, for lanes that `counts` (the others have no weight, whatever their finite scores); scores beyond the offset are looked for among the weights, those above
  // 2^kRaise, in the order of their bits (a NaN is above; an offset that no key has set yet, -inf, makes any weight infinite or a NaN).
  __device__ __forceinline__ void weights_of(const f32x4 (&s)[2], f32x4 (&w)[2], float scale_log2e, bool counts) {
    auto all = [&] {
      const float mu = counts ? m : INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale_log2e, -mu));
    };
    all();
    auto bits = [&](int t, int i) { return __float_as_uint(w[t][i]); };
    uint32_t most = max(max(bits(0, 0), bits(0, 1)), bits(0, 2));
    most = max(max(most, bits(0, 3)), bits(1, 0));
    most = max(max(most, bits(1, 1)), bits(1, 2));
    most = max(most, bits(1, 3));
    if (__any(most > __float_as_uint(256.f))) {
      raise(counts ? fmaxf(largest(s) * scale_log2e, kLowest) : -INFINITY);
      all();
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) l += (w[t][0] + w[t][1]) + (w[t][2] + w[t][3]);
  }
};

// Eight weights in two bf16 parts, the second never zero.
__device__ __forceinline__ void in_parts(const f32x4 (&p)[2], bf16x8 (&part)[2]) {
  uint32_t high[4], low[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = p[i >> 1][2 * (i & 1)], y = p[i >> 1][2 * (i & 1) + 1];
    high[i] = pack_bf16x2(x * (127.f / 128.f), y * (127.f / 128.f));
    low[i] = pack_bf16x2(x - __uint_as_float(high[i] << 16), y - __uint_as_float(high[i] & 0xffff0000u));
  }
  part[0] = __builtin_bit_cast(bf16x8, u32x4{high[0], high[1], high[2], high[3]});
  part[1] = __builtin_bit_cast(bf16x8, u32x4{low[0], low[1], low[2], low[3]});
}

// A list's blocks that hold keys, one after the other: `id` of a lane's entry, `slots` of them with keys, `left` whose are still to come.
struct Entries {
  int id, slots;
  unsigned long long left;
  // 0 slots: there is none
  __device__ __forceinline__ void pop(int& block, int& n) {
    n = 0;
    if (!left) return;  // (`block` stays: a block there is)
    const int l = __builtin_ctzll(left);
    left &= left - 1;
    block = __builtin_amdgcn_readlane(id, l);
    n = __builtin_amdgcn_readlane(slots, l);
  }
};

// bf16, head sizes up to 32 KS.
template <typename E, int KS>
struct Walk {
  static constexpr int X = 8, NK = KS, NV = 2 * KS, kLds = KS * 2048;  // bytes of LDS of a wavefront: 32 KS channels of 64 bytes
  u32x4 k[2][KS], v[2][KS];
  int block[2], n[2];

  // rows r < 8 of a score product are keys of the first block, the others of the second
  __device__ __forceinline__ void ask_k(const char* kbase, size_t stride, int D, int col, int quad) {
    const char* const at = kbase + (size_t)(col < 8 ? block[0] : block[1]) * stride;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const int unit = 4 * j + quad, slot = 8 * (col >> 2 & 1) + 4 * t + (col & 3);
        k[t][j] = *reinterpret_cast<const u32x4*>(at + ((j < KS - 1 || unit * X < D ? unit : 0) * 16 + slot) * 16);
      }
  }
  __device__ __forceinline__ void ask_v(const char* vbase, size_t stride, int D, int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* const at = vbase + (size_t)block[b] * stride;
#pragma unroll
      for (int i = 0; i < KS; ++i) v[b][i] = *reinterpret_cast<const u32x4*>(at + (i < KS - 1 || i * 64 + lane < 2 * D ? i * 64 + lane : 0) * 16);
    }
  }
  __device__ __forceinline__ void run(Entries list, const char* kbase, const char* vbase, size_t stride, int D, const u32x4 (&q)[NK], State<NV>& st, char* lds,
                                      int lane, int col, int quad, float scale_log2e) {
    block[0] = 0;
    list.pop(block[0], n[0]);
    block[1] = block[0];
    list.pop(block[1], n[1]);
    if (!n[0]) return;
    ask_k(kbase, stride, D, col, quad);
    ask_v(vbase, stride, D, lane);
    for (;;) {
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      if (4 * (KS - 1) * X + quad * X >= D)  // (channels that there are not: whatever was read in their place is no number to multiply)
#pragma unroll
        for (int t = 0; t < 2; ++t) k[t][KS - 1] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][j]), __builtin_bit_cast(bf16x8, q[j]), s[t], 0, 0, 0);
      const int had[2] = {n[0], n[1]};
      list.pop(block[0], n[0]);
      if (n[0]) block[1] = block[0];
      list.pop(block[1], n[1]);
      ask_k(kbase, stride, D, col, quad);  // (behind the last ones: those once more)
      if (had[0] + had[1] < 32) {
        // slots without a key: no weight, and their values (stale bits, possibly NaN) must not meet a zero weight
        const int here = quad < 2 ? had[0] : had[1];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (8 * (quad & 1) + 4 * t + i >= here) s[t][i] = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int slot = 8 * (lane & 1) + 2 * w;
              v[b][i][w] &= (slot < had[b] ? 0xffffu : 0u) | (slot + 1 < had[b] ? 0xffff0000u : 0u);
            }
      }
      // channel d: 64 bytes, a unit of 16 for each half of each block, at unit ^ (d >> 2 & 3)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const int d = i * 32 + (lane >> 1);
          *reinterpret_cast<u32x4*>(lds + d * 64 + ((2 * b + (lane & 1)) ^ (d >> 2 & 3)) * 16) = v[b][i];
        }
      ask_v(vbase, stride, D, lane);
      st.weights(s, scale_log2e);
      bf16x8 part[2];
      in_parts(s, part);
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) {
        const int d = dt * 16 + col;
        const bf16x8 x = *reinterpret_cast<const bf16x8*>(lds + d * 64 + (quad ^ (d >> 2 & 3)) * 16);
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, part[0], st.o[dt], 0, 0, 0);
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, part[1], st.o[dt], 0, 0, 0);
      }
      if (!n[0]) return;
    }
  }
};

// fp32, head sizes up to 32 KS.
template <int KS>
struct Walk<float, KS> {
  static constexpr int X = 4, NK = 2 * KS, NV = 2 * KS, kLds = 0, kDepth = KS <= 2 ? 3 : KS <= 6 ? 2 : 1;  // (as many blocks as fit in the registers)
  struct Block {
    u32x4 k[NK];
    f32x4 v[NV];
    int n;
  } ring[kDepth];

  __device__ __forceinline__ void run(Entries list, const char* kbase, const char* vbase, size_t stride, int D, const u32x4 (&q)[NK], State<NV>& st, char*, int lane,
                                      int col, int quad, float scale_log2e) {
    auto fetch = [&](Block& o) {
      int at = 0;
      list.pop(at, o.n);
      // (none: the descriptors end where they begin, and the loads touch no memory)
      const int bytes = o.n ? 64 * D : 0;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kbase) + at * stride, 0, bytes, kRsrc);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vbase) + at * stride, 0, bytes, kRsrc);
#pragma unroll
      for (int j = 0; j < NK; ++j) o.k[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, lane * 16 + j * 1024, 0, 0));
#pragma unroll
      for (int dt = 0; dt < NV; ++dt)
        o.v[dt] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, col * 64 + quad * 16 + dt * 1024, 0, 0));
    };
    auto attend = [&](Block& o) {
      f32x4 s[1] = {{0.f, 0.f, 0.f, 0.f}}, t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const f32x4 a = __builtin_bit_cast(f32x4, o.k[j]), b = __builtin_bit_cast(f32x4, q[j]);
        s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], b[0], s[0], 0, 0, 0);
        t = __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], b[1], t, 0, 0, 0);
        s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[2], b[2], s[0], 0, 0, 0);
        t = __builtin_amdgcn_mfma_f32_16x16x4f32(a[3], b[3], t, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][i] += t[i];
      if (o.n < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * quad + i >= o.n) {
            s[0][i] = -INFINITY;
#pragma unroll
            for (int dt = 0; dt < NV; ++dt) o.v[dt][i] = 0.f;
          }
      }
      st.weights(s, scale_log2e);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int dt = 0; dt < NV; ++dt) st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(o.v[dt][e], s[0][e], st.o[dt], 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kDepth; ++i) fetch(ring[i]);
    for (bool more = true; more;) {
#pragma unroll
      for (int i = 0; i < kDepth; ++i) {
        if (ring[i].n == 0) {
          more = false;
          break;
        }
        attend(ring[i]);
        fetch(ring[i]);
      }
    }
  }
};

__device__ __forceinline__ void store4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(uint16_t* p, const f32x4& v) { *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

// The result of a row: o / l and the log of the sum of its weights; without keys (m -inf) 0 and -inf; of keys that all score -inf (l 0) 0 / 0.
template <typename E>
__device__ __forceinline__ void store_row(E* out, f32x4 o, float m, float l) {
  const bool none = m == -INFINITY;
  const float inv = l == 0.f ? NAN : 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = none ? 0.f : o[i] * inv;
  store4(out, o);
}
__device__ __forceinline__ float row_lse(float m, float l) { return m == -INFINITY ? m : l == 0.f ? NAN : (m + log2f(l)) * kLn2; }

// Workgroup x: K/V head x % Hkv, then part, then token, from t0 on.  With several parts: counters [T][Hkv] are zero and stay so.
template <typename E, int KS>
__global__ __launch_bounds__(kWaves * 64) void attn_sparse_kernel(const E* __restrict__ q, int q_row_stride, const E* __restrict__ k_cache,
                                                                   const E* __restrict__ v_cache, const int32_t* __restrict__ cu_q,
                                                                   const int32_t* __restrict__ ctx_before, const int32_t* __restrict__ block_table, int bt_stride,
                                                                   const int32_t* __restrict__ blocks, int num_selected, E* __restrict__ out,
                                                                   float* __restrict__ lse, float* states, uint32_t* counters, int B, int Hkv, int G, int D, int parts,
                                                                   int t0, float scale_log2e) {
  typedef Walk<E, KS> W;
  constexpr int NV = W::NV, NK = W::NK, X = W::X, kRow = 32 * KS + 4;
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ int s_order;
  // the walks', then the states [kWaves - 1][G][kRow]
  constexpr int kStates = (kWaves - 1) * kMaxGroup * kRow * 4, kWalks = kWaves * W::kLds;
  __shared__ __attribute__((aligned(16))) char s_any[kStates > kWalks ? kStates : kWalks];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
  const int g = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, part = rest % parts, t = t0 + rest / parts;
  int b = t, p;
  if (cu_q) {
    const SeqOf seq = find_sequence(cu_q, ctx_before, B, t, [](int cu, int) { return (long long)cu; });
    if (t - seq.tok0 >= seq.S) return;  // (behind the last sequence)
    b = seq.b;
    p = seq.cb + t - seq.tok0;
  } else {
    p = ctx_before[b];
  }
  const int last = p < 0 ? -1 : p >> 4;  // the last block with keys
  const int per_part = (num_selected + parts - 1) / parts, e0 = part * per_part, e1 = min(num_selected, e0 + per_part);
  const int32_t* const list = blocks + ((int64_t)t * Hkv + g) * num_selected;
  const int32_t* const table = block_table + (size_t)b * bt_stride;

  u32x4 qf[NK];
  const E* const qrow = q + (size_t)t * q_row_stride + (size_t)(g * G + min(col, G - 1)) * D;
#pragma unroll
  for (int j = 0; j < NK; ++j) {
    const int d = (4 * j + quad) * X;
    qf[j] = d < D ? *reinterpret_cast<const u32x4*>(qrow + d) : u32x4{0u, 0u, 0u, 0u};
  }
  State<NV> st;
#pragma unroll
  for (int dt = 0; dt < NV; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const size_t piece = (size_t)16 * D * sizeof(E);
  W walk;
  for (int first = e0 + wave; first < e1; first += kWaves * 64) {
    // 64 entries at a time, a lane each: which hold keys, their blocks and how many slots of them
    const int entry = first + kWaves * lane, j = entry < e1 ? list[entry] : -1;
    const bool has = j >= 0 && j <= last;
    const Entries mine = {has ? table[j] : 0, j == last ? (p & 15) + 1 : 16, __ballot(has)};
    walk.run(mine, reinterpret_cast<const char*>(k_cache) + g * piece, reinterpret_cast<const char*>(v_cache) + g * piece, Hkv * piece, D, qf, st,
             s_any + wave * W::kLds, lane, col, quad, scale_log2e);
  }
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  if (quad == 0) s_m[wave][col] = st.m, s_l[wave][col] = st.l;
  float* const s_acc = reinterpret_cast<float*>(s_any);
  if (W::kLds > 0) __syncthreads();  // (where the walks had their values)
  if (wave > 0 && col < G) {
    float* const mine = s_acc + ((size_t)(wave - 1) * G + col) * kRow + quad * 4;
#pragma unroll
    for (int dt = 0; dt < NV; ++dt) *reinterpret_cast<f32x4*>(mine + dt * 16) = st.o[dt];
  }
  __syncthreads();
  const size_t row0 = (size_t)t * (Hkv * G) + g * G;  // the first query head's row of the results
  const int slot_words = D + 4;                       // of a state: o, m, l and two that keep 16 bytes aligned; states [rows][parts]
  float* const my_states = states + row0 * parts * slot_words;
  const int range = G * parts * slot_words * 4;
  if (wave == 0 && col < G) {
    // the first wavefront adds the others' states to its own
    float M = st.m;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][col]);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = s_m[w][col], f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
      total += s_l[w][col] * f;
      const float* const theirs = s_acc + ((size_t)max(w - 1, 0) * G + col) * kRow + quad * 4;
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) {
        const f32x4 x = w == 0 ? st.o[dt] : *reinterpret_cast<const f32x4*>(theirs + dt * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[dt][i] = w == 0 ? x[i] * f : (mw == -INFINITY ? st.o[dt][i] : st.o[dt][i] + x[i] * f);
      }
    }
    if (parts == 1) {
      E* const to = out + (row0 + col) * D + quad * 4;
#pragma unroll
      for (int dt = 0; dt < NV; ++dt)
        if (dt * 16 + quad * 4 < D) store_row(to + dt * 16, st.o[dt], M, total);
      if (lse && quad == 0) lse[row0 + col] = row_lse(M, total);
    } else {
      const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(my_states, 0, range, kRsrc);
      const int at = (col * parts + part) * slot_words * 4;
#pragma unroll
      for (int dt = 0; dt < NV; ++dt)
        if (dt * 16 + quad * 4 < D) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, st.o[dt]), to, at + (dt * 16 + quad * 4) * 4, 0, kAgent);
      if (quad == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(M), __float_as_uint(total)}, to, at + D * 4, 0, kAgent);
    }
  }
  if (parts == 1) return;
  // the workgroup that is done last with the list adds the parts up, in their order: a wavefront to each query head, four elements a lane, several parts at a time
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the states are where every XCD finds them)
  __syncthreads();
  if (tid == 0) {
    uint32_t* const counter = counters + (size_t)t * Hkv + g;
    s_order = (int)__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (s_order == parts - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (__builtin_amdgcn_readfirstlane(s_order) != parts - 1) return;
  const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(my_states, 0, range, kRsrc);
  constexpr int kLanes = KS <= 2 ? 16 : KS <= 4 ? 32 : 64, kAtOnce = 64 / kLanes;  // lanes of a head vector, parts that a wavefront reads side by side
  const int el = lane % kLanes * 4, side = lane / kLanes;
  for (int h = wave; h < G; h += kWaves) {
    // (lane k: part k's m and l; at most 64 parts)
    const u32x2 ml = __builtin_amdgcn_raw_buffer_load_b64(from, (h * parts + min(lane, parts - 1)) * slot_words * 4 + D * 4, 0, kAgent);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const float mine = lane < parts ? __uint_as_float(ml[0]) : -INFINITY;
    const float M = wave_max(mine), f = mine == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine - M), total = wave_sum(lane < parts ? __uint_as_float(ml[1]) * f : 0.f);
    auto add_up = [&](auto ahead) {
      constexpr int kAhead = decltype(ahead)::value;
      for (int k0 = 0; k0 < parts; k0 += kAtOnce * kAhead) {
        f32x4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          x[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (h * parts + min(k0 + i * kAtOnce + side, parts - 1)) * slot_words * 4 + min(el, D - 4) * 4,
                                                                                 0, kAgent));
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int k = k0 + i * kAtOnce + side;
          const float w = __shfl(f, min(k, 63));
          if (k < parts)  // (also parts whose weight is 0: an infinite value there is no number times it)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += x[i][e] * w;
        }
      }
    };
    // (all parts at once, if registers allow; what there is not is asked for all the same: one token, 64 blocks in 8 parts, four at a time 9.9 us, sixteen 11.5; 256 in 32
    // 16.5 and 15.1)
    if (parts <= kAtOnce * 4) add_up(std::integral_constant<int, 4>());
    else if (parts <= kAtOnce * 8) add_up(std::integral_constant<int, 8>());
    else add_up(std::integral_constant<int, 16>());
#pragma unroll
    for (int s = kLanes; s < 64; s <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], s);
    if (side == 0 && el < D) store_row(out + (row0 + h) * D + el, o, M, total);
    if (lse && lane == 0) lse[row0 + h] = row_lse(M, total);
  }
}

// Prompts, bf16: sixteen (eight) wavefronts have the tokens of a group, two (one) each and side by side in the columns (their heads padded to a power of two), and walk the
// union of the group's lists, eight (four) blocks at a time through LDS, each for the blocks that its own tokens list.  A column whose token does not list a block
// has no weight there.
//   The union: a word per block of the sequence with a bit per token, from which the listed ones are collected in their order.
//   Where that does not do, the wavefront takes its tokens one by one, block by block: lists with a block twice, and results that are not
// finite (a NaN or an infinity among values meets the zero weights of the columns beside it).  That loop goes through scratch memory for what the registers do not hold (up to 37 of them;
// the main loop does not).
//   The weights go in two bf16 parts here too, so that what a token gets does not depend on the tokens beside it or on the table's width (one part, 8 bits: 120 us,
// so 145; but 1.4 times the error that the result's rounding leaves).
//   Blocks go from memory into LDS without registers between, and the operands of a pair of blocks are asked for together, half of the values' before the weights are known
// (with weights in one part: in registers, operands as they are wanted: 145 us, so 131; values all at once: 140).
// What bounds it (895 tokens, 64 heads on 8 of 128, lists of 64 that agree in half): latency.  A workgroup fills a CU, its wavefronts leave a barrier together, and want
// LDS, the matrix unit and the vector unit at the same times, which are busy for 27, 25 and 39% of it; at a barrier they wait for the one with the most blocks of a stage (the
// sum of those is 1.7 times the mean's), and the workgroup with the largest union comes last.  A column's work is in vain for 40% of a wavefront's blocks, those that the token
// beside it lists alone.  Token by token the same call reads each block of K and V 20 times from the caches, 3.7 GB, 235 us.
constexpr int kWords = 5120;  // blocks of a sequence that the union has room for
constexpr int group_waves(int KS) { return KS <= 4 ? 16 : 8; }  // (as many as have the registers)
// Tokens of a wavefront.
constexpr int tokens_of_wave(int log_rows) { return log_rows >= 4 ? 1 : 2; }

template <int KS>
__global__ __launch_bounds__(group_waves(KS) * 64, group_waves(KS) / 4) void attn_sparse_prompt_kernel(
    const uint16_t* __restrict__ q, int q_row_stride, const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ ctx_before, const int32_t* __restrict__ block_table, int bt_stride, const int32_t* __restrict__ blocks, int num_selected,
    uint16_t* __restrict__ out, float* __restrict__ lse, int B, int Hkv, int G, int log_rows, int D, int unit0, float scale_log2e) {
  constexpr int NV = 2 * KS, kPiece = KS * 1024;  // a block's K or V in LDS: channels up to 32 KS
  constexpr int kEarly = NV < 4 ? NV : 4;         // of a pair of blocks' values, how much is asked for before the weights are known (registers)
  constexpr int kGroupWaves = group_waves(KS), kStage = kGroupWaves / 2, words = kWords;  // a wavefront to each piece of a stage's blocks
  __shared__ __attribute__((aligned(16))) char s_stage[2 * kStage * 2 * kPiece];  // twice kStage blocks, K and V
  __shared__ uint32_t s_word[words];
  __shared__ uint16_t s_list[words];
  __shared__ int s_count[kGroupWaves], s_alone;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
  const int g = blockIdx.x % Hkv, unit = unit0 + blockIdx.x / Hkv, per_wave = tokens_of_wave(log_rows), group = kGroupWaves * per_wave;
  auto first_unit = [&](int cu, int s) { return (long long)(cu / group) + s; };
  const SeqOf seq = find_sequence(cu_q, ctx_before, B, unit, first_unit);
  const int i0 = (int)(unit - first_unit(seq.tok0, seq.b)) * group, n = min(group, seq.S - i0);
  if (n <= 0) return;
  const int first = seq.tok0 + i0, p0 = seq.cb + i0;  // the group's first token and its position
  const int32_t* const table = block_table + (size_t)seq.b * bt_stride;

  // the union of the lists
  for (int i = tid; i < words; i += kGroupWaves * 64) s_word[i] = 0;
  if (tid == 0) s_alone = 0;
  __syncthreads();
  bool alone = false;
  for (int t = wave; t < n; t += kGroupWaves) {
    const int last = p0 + t < 0 ? -1 : (p0 + t) >> 4;
    const int32_t* const list = blocks + ((int64_t)(first + t) * Hkv + g) * num_selected;
    for (int i = lane; i < num_selected; i += 64) {
      const int j = list[i];
      if (j < 0 || j > last) continue;
      if (j >= words) alone = true;  // (cannot be: the launch has looked at the table's width)
      else alone |= (atomicOr(&s_word[j], 1u << t) >> t & 1u) != 0;
    }
  }
  if (alone) s_alone = 1;
  __syncthreads();
  int listed = 0;
  if (!s_alone) {
    // a run of words to each wavefront
    const int run = (words + kGroupWaves * 64 - 1) / (kGroupWaves * 64) * 64, w0 = wave * run, w1 = min(words, w0 + run);
    int mine = 0;
    for (int i = w0; i < w1; i += 64) mine += __popcll(__ballot(i + lane < w1 && s_word[i + lane] != 0));
    if (lane == 0) s_count[wave] = mine;
    __syncthreads();
    int at = 0;
    for (int w = 0; w < kGroupWaves; ++w) {
      at += w < wave ? s_count[w] : 0;
      listed += s_count[w];
    }
    for (int i = w0; i < w1; i += 64) {
      const unsigned long long m = __ballot(i + lane < w1 && s_word[i + lane] != 0);
      if (m >> lane & 1) s_list[at + __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u))] = (uint16_t)(i + lane);
      at += __popcll(m);
    }
    __syncthreads();
  }

  // this wavefront's columns: head col % rows of its token col / rows
  const int rows = 1 << log_rows, mine0 = wave * per_wave, have = min(per_wave, n - mine0);
  const int tok = min(col >> log_rows, per_wave - 1), head = col & (rows - 1), p = p0 + mine0 + tok;
  const bool real = (col >> log_rows) < have && head < G;
  const size_t piece = (size_t)16 * D * 2, stride = Hkv * piece;
  const char *const kbase = reinterpret_cast<const char*>(k_cache) + g * piece, *const vbase = reinterpret_cast<const char*>(v_cache) + g * piece;
  auto ask_q = [&](u32x4 (&qf)[KS], int token, int h) {
    const uint16_t* const row = q + (size_t)token * q_row_stride + (size_t)(g * G + h) * D;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[j] = (4 * j + quad) * 8 < D ? *reinterpret_cast<const u32x4*>(row + (4 * j + quad) * 8) : u32x4{0u, 0u, 0u, 0u};
  };
  u32x4 qf[KS];
  ask_q(qf, first + min(mine0 + tok, n - 1), min(head, G - 1));
  State<NV> st;
#pragma unroll
  for (int dt = 0; dt < NV; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t k_place = quad * 256 + (8 * (col >> 2 & 1) + (col & 3)) * 16, v_place = kPiece + col * 32 + (quad & 1) * 16;
  const uint32_t my_bits = have > 0 ? ((1u << have) - 1u) << mine0 : 0u, my_bit = real ? 1u << (mine0 + tok) : 0u;
  // Two blocks in LDS, K and then V, at a and b.  `counts`: the column's token lists the lane's one (quads 0 and 1: a); if some lane sees not all of its 16 keys
  // (`ragged`), seen() of them.  (kOne: the first block alone, the second's values do not count at all)
  const uint32_t half_k = col < 8 ? 0u : ~0u, half_v = quad < 2 ? 0u : ~0u;
  auto attend = [&](auto one, uint32_t a, uint32_t b, bool counts, auto seen, bool ragged) {
    constexpr bool kOne = decltype(one)::value;
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    const char* const kat = s_stage + (a + (half_k & (b - a)) + k_place);
    u32x4 x[KS][2];
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) x[j][t] = *reinterpret_cast<const u32x4*>(kat + j * 1024 + t * 64);
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[j][t]), __builtin_bit_cast(bf16x8, qf[j]), s[t], 0, 0, 0);
    const char* const vat = s_stage + (a + (half_v & (b - a)) + v_place);
    u32x4 y[NV];
#pragma unroll
    for (int dt = 0; dt < kEarly; ++dt) y[dt] = *reinterpret_cast<const u32x4*>(vat + dt * 512);
    if (ragged) {
      const int n = seen();
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = 8 * (quad & 1) + 4 * t + e < n ? s[t][e] : -INFINITY;
    }
    f32x4 p[2];
    st.weights_of(s, p, scale_log2e, counts);
    bf16x8 part[2];
    in_parts(p, part);
    __builtin_amdgcn_s_setprio(1);  // (wavefronts that multiply go before those that count: 152 -> 142 us)
#pragma unroll
    for (int dt = kEarly; dt < NV; ++dt) y[dt] = *reinterpret_cast<const u32x4*>(vat + dt * 512);
#pragma unroll
    for (int dt = 0; dt < NV; ++dt) {
      if (kOne && quad >= 2) y[dt] = u32x4{0u, 0u, 0u, 0u};
      st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y[dt]), part[0], st.o[dt], 0, 0, 0);
      st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y[dt]), part[1], st.o[dt], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // K or V of a block, from memory to LDS by a wavefront
  auto bring = [&](const char* at, uint32_t to) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int u = k * 64 + lane;
      __builtin_amdgcn_global_load_lds((gptr_t)(at + (k < KS - 1 || u < 2 * D ? u : 0) * 16), (lptr_t)(s_stage + to + k * 1024), 16, 0, 0);
    }
  };
  // ... once it is there: channels of K that there are not, and values behind the last token (stale bits, possibly NaN), must not meet zeros of the other side
  auto arrived = [&](uint32_t at, bool is_v, int slots) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    char* const mine = s_stage + at + lane * 16;
    if (!is_v && D != 32 * KS && (KS - 1) * 64 + lane >= 2 * D) *reinterpret_cast<u32x4*>(mine + (KS - 1) * 1024) = u32x4{0u, 0u, 0u, 0u};
    if (is_v && slots < 16) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32x4 x = *reinterpret_cast<const u32x4*>(mine + k * 1024);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int slot = 8 * (lane & 1) + 2 * w;
          x[w] &= (slot < slots ? 0xffffu : 0u) | (slot + 1 < slots ? 0xffff0000u : 0u);
        }
        *reinterpret_cast<u32x4*>(mine + k * 1024) = x;
      }
    }
  };
  // the wavefront's piece of a stage is of the block list[i + wave / 2]; its place in memory is known a stage before it is asked for
  auto index_of = [&](int i) { return __builtin_amdgcn_readfirstlane(s_list[min(i + (wave >> 1), listed - 1)]); };
  int j_ask = 0, id_ask = 0, slots_next = 16;
  auto ask = [&](int i) {
    bring((wave & 1 ? vbase : kbase) + (size_t)id_ask * stride, (i / kStage & 1) * (kStage * 2 * kPiece) + wave * kPiece);
    slots_next = min(16, p0 + n - j_ask * 16);
    j_ask = index_of(i + kStage);  // (behind the last ones: the last one)
    id_ask = table[j_ask];
  };
  // a stage's blocks and the tokens that list them, a lane each
  int j_here = 0;
  uint32_t bits_here = 0;
  auto look = [&](int i) {
    j_here = s_list[min(i + (lane & (kStage - 1)), listed - 1)];
    bits_here = s_word[j_here];
  };
  if (listed > 0) {
    j_ask = index_of(0);
    id_ask = table[j_ask];
    ask(0);
    look(0);
  }
  for (int i = 0; i < listed; i += kStage) {
    const uint32_t buf = (i / kStage & 1) * (kStage * 2 * kPiece);
    arrived(buf + wave * kPiece, wave & 1, slots_next);
    __syncthreads();  // (who has passed it is through with the blocks before the last ones: one barrier a turn)
    ask(i + kStage);
    // the blocks that tokens of this wavefront list, two at a time
    const int j_now = j_here;
    const uint32_t bits_now = bits_here;
    unsigned long long want = __ballot(lane < kStage && i + lane < listed && (bits_now & my_bits) != 0);
    look(i + kStage);
    while (want) {
      const int a = __builtin_ctzll(want);
      want &= want - 1;
      const bool pair = want != 0;
      const int b = pair ? __builtin_ctzll(want) : a;
      want &= want - 1;
      const int ja = __builtin_amdgcn_readlane(j_now, a), jb = __builtin_amdgcn_readlane(j_now, b);
      const uint32_t ba = __builtin_amdgcn_readlane(bits_now, a), bb = pair ? __builtin_amdgcn_readlane(bits_now, b) : 0u;
      // the column's token lists the lane's block, and sees its keys: all, but for blocks that a token of the group is in
      attend(std::false_type(), buf + a * (2 * kPiece), buf + b * (2 * kPiece), ((ba ^ (half_v & (ba ^ bb))) & my_bit) != 0,
             [&] { return p + 1 - (quad < 2 ? ja : jb) * 16; }, max(ja, jb) >= p0 >> 4);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what was brought in for a stage behind the last)
  __syncthreads();                                  // (all wavefronts are through with the stages)
  auto finish = [&](int token, int h, bool store) {
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    if (!store) return;
    const size_t row = (size_t)token * (Hkv * G) + g * G + h;
#pragma unroll
    for (int dt = 0; dt < NV; ++dt)
      if (dt * 16 + quad * 4 < D) store_row(out + row * D + dt * 16 + quad * 4, st.o[dt], st.m, st.l);
    if (lse && quad == 0) lse[row] = row_lse(st.m, st.l);
  };
  float odd = 0.f;  // not a number once a sum is not finite
#pragma unroll
  for (int dt = 0; dt < NV; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (dt * 16 + quad * 4 < D) odd = __builtin_fmaf(st.o[dt][e], 0.f, odd);
  if (!s_alone && !__any(odd != odd)) {
    finish(first + mine0 + tok, head, real);
    return;
  }
  // token by token
  for (int t = 0; t < have; ++t) {
    const int token = first + mine0 + t, at = p0 + mine0 + t, last = at < 0 ? -1 : at >> 4;
    ask_q(qf, token, min(col, G - 1));
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int dt = 0; dt < NV; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int32_t* const list = blocks + ((int64_t)token * Hkv + g) * num_selected;
    const uint32_t own = wave * (2 * kPiece);
    for (int i = 0; i < num_selected; ++i) {
      const int j = __builtin_amdgcn_readfirstlane(list[i]);
      if (j < 0 || j > last) continue;
      const size_t block = (size_t)table[j] * stride;
      const int slots = min(16, at + 1 - j * 16);
      bring(kbase + block, own);
      bring(vbase + block, own + kPiece);
      arrived(own, false, 16);
      arrived(own + kPiece, true, slots);
      attend(std::true_type(), own, own, quad < 2, [&] { return slots; }, true);
    }
    finish(token, col, col < G);
  }
}

// Prompts of so many rows that the groups' lists in common save more than a group's walk, which takes 115 us of 64 blocks, alone or beside others, costs.  (us of a call, token
// by token / groups: 64 on 8, 128, lists of 64: 256 tokens 66 / 126, 512 128 / 141 (behind 2000 tokens 126 / 95), 700 175 / 148, 4 x 512 479 / 270, 8 x 48 97 / 103; 2000, of 32,
// 300 / 182; 52 on 52: 32 95 / 118, 64 185 / 120, 128 380 / 127; 32 on 8, 64: 512 65 / 113, 1024 133 / 121, 4 x 512 266 / 207; 8 on 1, 4 x 512 70 / 124; 8 on 1, 256: 1024 97 / 183,
// 4 x 512 183 / 164, 2000, of 32, 128 / 113.  The line is drawn in channels of K rows; 64 tokens of 52 on 52 and the last one are on its wrong side.)
struct SparseGroups {
  int log_rows, units;  // units 0: token by token
  explicit operator bool() const { return units > 0; }
};
SparseGroups sparse_groups(const SparseArgs& a) {
  int log_rows = 0;
  while (a.Hkv << log_rows < a.Hq) ++log_rows;
  const int group = group_waves((a.D + 31) / 32) * tokens_of_wave(log_rows);
  const bool many = a.cu_q && (int64_t)a.T * a.Hkv * a.D >= 2048 * (int64_t)a.num_cu && a.T / a.B >= group && a.bt_stride <= kWords;
  return {log_rows, many ? a.T / group + a.B : 0};
}
// n units of `wgs` workgroups of so many threads: launches of fewer than 2^32 threads each.
template <typename F>
void in_launches(int n, int wgs, int threads, F f) {
  const int most = std::max(1, (int)(((int64_t)1 << 31) / threads / wgs));
  for (int64_t u = 0; u < n; u += most) f((int)u, std::min(most, (int)(n - u)));
}

template <int KS>
void launch_groups(const SparseArgs& a, const SparseGroups& by, hipStream_t s) {
  in_launches(by.units, a.Hkv, group_waves(KS) * 64, [&](int unit0, int units) {
    hipLaunchKernelGGL((attn_sparse_prompt_kernel<KS>), dim3((unsigned)(a.Hkv * units)), dim3(group_waves(KS) * 64), 0, s, (const uint16_t*)a.q, a.q_row_stride,
                       (const uint16_t*)a.k_cache, (const uint16_t*)a.v_cache, a.cu_q, a.ctx_before, a.block_table, a.bt_stride, a.blocks, a.num_selected, (uint16_t*)a.out,
                       a.lse, a.B, a.Hkv, a.Hq / a.Hkv, by.log_rows, a.D, unit0, a.scale_log2e);
  });
}

template <typename E, int KS>
void launch_steps(const SparseArgs& a, hipStream_t s) {
  if constexpr (std::is_same<E, uint16_t>::value) {
    if (const SparseGroups by = sparse_groups(a)) return launch_groups<KS>(a, by, s);
  }
  const int G = a.Hq / a.Hkv, parts = sparse_parts(a.Hkv, a.T, a.num_selected, a.num_cu, a.dtype);
  in_launches(a.T, a.Hkv * parts, kWaves * 64, [&](int t0, int tokens) {
    hipLaunchKernelGGL((attn_sparse_kernel<E, KS>), dim3((unsigned)(a.Hkv * parts * tokens)), dim3(kWaves * 64), 0, s, (const E*)a.q, a.q_row_stride,
                       (const E*)a.k_cache, (const E*)a.v_cache, a.cu_q, a.ctx_before, a.block_table, a.bt_stride, a.blocks, a.num_selected, (E*)a.out, a.lse, a.states,
                       a.counters, a.B, a.Hkv, G, a.D, parts, t0, a.scale_log2e);
  });
}

template <typename E>
void launch_typed(const SparseArgs& a, hipStream_t s) {
  switch ((a.D + 31) / 32) {
    case 1: return launch_steps<E, 1>(a, s);
    case 2: return launch_steps<E, 2>(a, s);
    case 3: return launch_steps<E, 3>(a, s);
    case 4: return launch_steps<E, 4>(a, s);
    case 5: return launch_steps<E, 5>(a, s);
    case 6: return launch_steps<E, 6>(a, s);
    case 7: return launch_steps<E, 7>(a, s);
    default: return launch_steps<E, 8>(a, s);
  }
}

}  // namespace

hipError_t launch_attn_sparse(const SparseArgs& a, hipStream_t s) {
  if (a.dtype == ECOSERVE_BF16) launch_typed<uint16_t>(a, s);
  else launch_typed<float>(a, s);
  return hipGetLastError();
}

}  // namespace eco
