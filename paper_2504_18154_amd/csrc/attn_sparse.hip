// Attention over listed blocks of the paged cache (Eq. 2 of Section 2.1 over the keys of the blocks in a list), for decode
// steps and prompts alike: every (token, K/V head) has a list of its own.
//
// The unit of work is one (token, K/V head): its G query heads are the columns of the products, the cache blocks in its list
// come in operand layout as everywhere in this library (see attn_any_mfma.hip):
//   scores  S^T[key][head] = K . Q^T      values  O^T[d][head] += V^T . P^T
// fp32: v_mfma_f32_16x16x4_f32; bf16: v_mfma_f32_16x16x32_bf16 and v_mfma_f32_16x16x16_bf16, the weights in two bf16 parts (16 bits).
// The first part is the weight less 1/128 of it, so that the second is never zero: a value that is infinite meets two weights that are not.
//
// A workgroup of four wavefronts has one list, or a part of it where there are few; the wavefronts take its entries in turn, with the
// blocks of the next entries on their way (entries without keys are dropped before any load).  Their states are added up through LDS,
// those of parts by a second launch.  Bound by reading K and V: from memory in a decode step, from the caches behind prompts, whose
// neighbouring tokens list much the same blocks; the K/V heads go to different XCDs (consecutive workgroups), so that an XCD's
// cache holds the blocks of one or a few.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "sparse.h"

namespace eco {

namespace {

constexpr int kWaves = 4;
constexpr int kRsrc = 0x00020000;  // buffer descriptor: untyped 32-bit data, no swizzle, no stride
constexpr float kRaise = 8.f;      // the exponent offset is raised when a score exceeds it by more (log2 units)

// A cache block as operands, head sizes up to 32 KS.
template <typename E, int KS>
struct Operands {
  static constexpr bool kF32 = std::is_same<E, float>::value;
  static constexpr int X = Elem<E>::X, NK = kF32 ? 2 * KS : KS, NV = 2 * KS;
  typedef typename std::conditional<kF32, f32x4, s16x4>::type VFrag;
  u32x4 k[NK];
  VFrag v[NV];
  int n;  // slots that hold keys; 0: no block

  // (no block: the descriptors end where they begin, and the loads touch no memory)
  __device__ __forceinline__ void load(const char* kbase, const char* vbase, int bytes, int lane, int col, int quad) {
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kbase), 0, bytes, kRsrc);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vbase), 0, bytes, kRsrc);
#pragma unroll
    for (int j = 0; j < NK; ++j) k[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, lane * 16 + j * 1024, 0, 0));
#pragma unroll
    for (int dt = 0; dt < NV; ++dt) {
      if constexpr (kF32) v[dt] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, col * 64 + quad * 16 + dt * 1024, 0, 0));
      else v[dt] = __builtin_bit_cast(s16x4, __builtin_amdgcn_raw_buffer_load_b64(rv, col * 32 + quad * 8 + dt * 512, 0, 0));
    }
  }

  // One step of the online softmax: m exponent offset (-inf: no key yet), l this lane's share of the sum, acc unnormalised.
  __device__ __forceinline__ void attend(const u32x4 (&q)[NK], float& m, float& l, f32x4 (&acc)[NV], int quad, float scale_log2e) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (kF32) {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const f32x4 a = __builtin_bit_cast(f32x4, k[j]), b = __builtin_bit_cast(f32x4, q[j]);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], b[0], s, 0, 0, 0);
        t = __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], b[1], t, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[2], b[2], s, 0, 0, 0);
        t = __builtin_amdgcn_mfma_f32_16x16x4f32(a[3], b[3], t, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += t[i];
    } else {
#pragma unroll
      for (int j = 0; j < NK; ++j)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[j]), __builtin_bit_cast(bf16x8, q[j]), s, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] *= scale_log2e;
    if (n < 16) {
      // slots without a key: no weight, and their values (stale bits, possibly NaN) must not meet a zero weight
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * quad + i >= n) s[i] = -INFINITY;
#pragma unroll
      for (int dt = 0; dt < NV; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * quad + i >= n) v[dt][i] = 0;
    }
    float bm = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    if (__any(bm > m + kRaise)) {
      bm = fmaxf(bm, __shfl_xor(bm, 16));
      bm = fmaxf(bm, __shfl_xor(bm, 32));
      const float m_new = bm > m + kRaise ? bm : m;
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < NV; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[dt][i] *= alpha;
      m = m_new;
    }
    const float mu = m == -INFINITY ? 0.f : m;
    f32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(s[i] - mu);
    l += (p[0] + p[1]) + (p[2] + p[3]);
    if constexpr (kF32) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int dt = 0; dt < NV; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt][e], p[e], acc[dt], 0, 0, 0);
    } else {
      f32x4 less;
#pragma unroll
      for (int i = 0; i < 4; ++i) less[i] = p[i] * (127.f / 128.f);
      const bf16x4 high = __builtin_convertvector(less, bf16x4);
      f32x4 left;
#pragma unroll
      for (int i = 0; i < 4; ++i) left[i] = p[i] - (float)high[i];
      const s16x4 part0 = __builtin_bit_cast(s16x4, high), part1 = __builtin_bit_cast(s16x4, __builtin_convertvector(left, bf16x4));
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[dt], part0, acc[dt], 0, 0, 0);
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[dt], part1, acc[dt], 0, 0, 0);
    }
  }
};

__device__ __forceinline__ void store4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(uint16_t* p, const f32x4& v) { *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

// The result of a row: o / l and the log of the sum of its weights; without keys 0 and -inf.
template <typename E>
__device__ __forceinline__ void store_row(E* out, f32x4 o, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = l == 0.f ? 0.f : o[i] * inv;
  store4(out, o);
}
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2; }

// Workgroup x: K/V head x % Hkv, then part, then token.
template <typename E, int KS, int DEPTH>
__global__ __launch_bounds__(kWaves * 64) void attn_sparse_kernel(const E* __restrict__ q, int q_row_stride, const E* __restrict__ k_cache,
                                                                   const E* __restrict__ v_cache, const int32_t* __restrict__ cu_q,
                                                                   const int32_t* __restrict__ ctx_before, const int32_t* __restrict__ block_table, int bt_stride,
                                                                   const int32_t* __restrict__ blocks, int num_selected, E* __restrict__ out,
                                                                   float* __restrict__ lse, float* __restrict__ states, int B, int T, int Hkv, int G, int D, int parts,
                                                                   float scale_log2e) {
  typedef Operands<E, KS> Op;
  constexpr int NV = Op::NV, NK = Op::NK, X = Op::X;
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  extern __shared__ __attribute__((aligned(16))) float s_acc[];  // [kWaves - 1][G][32 KS + 4]
  constexpr int kRow = 32 * KS + 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
  const int g = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, part = rest % parts, t = rest / parts;
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
  float m = -INFINITY, l = 0.f;
  f32x4 acc[NV];
#pragma unroll
  for (int dt = 0; dt < NV; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int piece = 16 * D * (int)sizeof(E);
  const char *const kbase = reinterpret_cast<const char*>(k_cache), *const vbase = reinterpret_cast<const char*>(v_cache);
  for (int first = e0 + wave; first < e1; first += kWaves * 64) {
    // 64 entries at a time, a lane each: which hold keys, their blocks and how many slots of them
    const int entry = first + kWaves * lane, j = entry < e1 ? list[entry] : -1;
    const bool has = j >= 0 && j <= last;
    const int id = has ? table[j] : 0, slots = j == last ? (p & 15) + 1 : 16;
    unsigned long long left = __ballot(has);
    Op op[DEPTH];
    auto fetch = [&](Op& o) {
      int at = 0, bytes = 0;
      o.n = 0;
      if (left) {
        const int l0 = __builtin_ctzll(left);
        left &= left - 1;
        at = __builtin_amdgcn_readlane(id, l0);
        o.n = __builtin_amdgcn_readlane(slots, l0);
        bytes = piece;
      }
      const size_t base = ((size_t)at * Hkv + g) * piece;
      o.load(kbase + base, vbase + base, bytes, lane, col, quad);
    };
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) fetch(op[i]);
    for (bool more = true; more;) {
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        if (op[i].n == 0) {
          more = false;
          break;
        }
        op[i].attend(qf, m, l, acc, quad, scale_log2e);
        fetch(op[i]);
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (quad == 0) s_m[wave][col] = m, s_l[wave][col] = l;
  if (wave > 0 && col < G) {
    float* const mine = s_acc + ((size_t)(wave - 1) * G + col) * kRow + quad * 4;
#pragma unroll
    for (int dt = 0; dt < NV; ++dt) *reinterpret_cast<f32x4*>(mine + dt * 16) = acc[dt];
  }
  __syncthreads();
  if (wave > 0 || col >= G) return;
  // the first wavefront adds the others' states to its own
  float M = m;
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
      const f32x4 x = w == 0 ? acc[dt] : *reinterpret_cast<const f32x4*>(theirs + dt * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[dt][i] = w == 0 ? x[i] * f : (mw == -INFINITY ? acc[dt][i] : acc[dt][i] + x[i] * f);
    }
  }
  const size_t row = (size_t)t * (Hkv * G) + g * G + col;
  if (parts == 1) {
#pragma unroll
    for (int dt = 0; dt < NV; ++dt)
      if (dt * 16 + quad * 4 < D) store_row(out + row * D + dt * 16 + quad * 4, acc[dt], total);
    if (lse && quad == 0) lse[row] = row_lse(M, total);
  } else {
    float* const state = states + ((size_t)part * T * (Hkv * G) + row) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < NV; ++dt)
      if (dt * 16 + quad * 4 < D) *reinterpret_cast<f32x4*>(state + dt * 16 + quad * 4) = acc[dt];
    if (quad == 0) state[D] = M, state[D + 1] = total;
  }
}

// One wavefront per (token, query head): the states of its parts.  A lane has four elements.
template <typename E>
__global__ __launch_bounds__(256) void merge_parts_kernel(const float* __restrict__ states, const int32_t* __restrict__ cu_q, int B, E* __restrict__ out,
                                                          float* __restrict__ lse, int64_t rows, int Hq, int D, int parts) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows || (cu_q && row / Hq >= cu_q[B])) return;
  const float* const first = states + row * (D + 4);
  const int64_t step = rows * (D + 4);
  // a lane's share of the parts' offsets and sums (at most 64 parts)
  const float mine = lane < parts ? first[lane * step + D] : -INFINITY;
  const float M = wave_max(mine), f = mine == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine - M);
  const float total = wave_sum(lane < parts ? first[lane * step + D + 1] * f : 0.f);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const bool in = lane * 4 < D;
  for (int k = 0; k < parts; ++k) {
    const float w = __shfl(f, k);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (in) x = *reinterpret_cast<const f32x4*>(first + k * step + lane * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = w == 0.f ? o[i] : o[i] + x[i] * w;
  }
  if (in) store_row(out + row * D + lane * 4, o, total);
  if (lse && lane == 0) lse[row] = row_lse(M, total);
}

template <typename E, int KS>
void launch_steps(const SparseArgs& a, hipStream_t s) {
  constexpr int kDepth = sizeof(E) * KS <= 8 ? 3 : sizeof(E) * KS <= 24 ? 2 : 1;  // (as many as fit in the registers)
  const int G = a.Hq / a.Hkv, parts = sparse_parts(a.Hkv, a.T, a.num_selected, a.num_cu);
  const size_t lds = (size_t)(kWaves - 1) * G * (32 * KS + 4) * sizeof(float);
  hipLaunchKernelGGL((attn_sparse_kernel<E, KS, kDepth>), dim3((unsigned)((int64_t)a.Hkv * parts * a.T)), dim3(kWaves * 64), lds, s, (const E*)a.q, a.q_row_stride,
                     (const E*)a.k_cache, (const E*)a.v_cache, a.cu_q, a.ctx_before, a.block_table, a.bt_stride, a.blocks, a.num_selected, (E*)a.out, a.lse, a.states,
                     a.B, a.T, a.Hkv, G, a.D, parts, a.scale_log2e);
  if (parts > 1) {
    const int64_t rows = (int64_t)a.T * a.Hq;
    hipLaunchKernelGGL((merge_parts_kernel<E>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a.states, a.cu_q, a.B, (E*)a.out, a.lse, rows, a.Hq, a.D, parts);
  }
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
