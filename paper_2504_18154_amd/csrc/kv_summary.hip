// Block summaries: of every channel of a full cache block the largest and the smallest key, in one byte each with one
// exponent for the (block, K/V head): what block_select.hip scores blocks by (layout in include/ecoserve.h).
//
// The exponent follows from the largest |key|, the codes are rounded outward, and scaling by a power of two is exact: the
// result does not depend on any order.  A wavefront takes one K/V head of one block: a lane brings in slots lane % 4, + 4,
// + 8, + 12 of one 16-byte unit (64 bytes in a row per four lanes), takes the extremes over them in registers and over its
// three neighbours within the vector unit.  The extremes are taken of whole numbers in the keys' order (x ^ 0x7fff.. where x is negative), two bf16 keys an
// instruction; NaNs lie beyond the infinities there, so that the extremes tell whether the block holds either.
// Memory bounds a prompt's blocks (each is read once, for 1/16 of it written; 65536 tokens, 8 heads of 128, 134 MB: 33 us from memory; 26 from the
// last-level cache, where floats took 28), latency a step's.
//
// Blocks are numbered sequence after sequence, those of sequence b from cu_q[b] / 16 + b: S new tokens fill at most
// S / 16 + 1 blocks.
#include <type_traits>

#include "common.h"
#include "summary.h"

namespace eco {

namespace {

constexpr int kSummaryThreads = 256;

// Keys as whole numbers in their order.  bf16: two in a word.
typedef short s16x2 __attribute__((ext_vector_type(2)));
template <typename E>
struct Order;
template <>
struct Order<uint16_t> {
  typedef s16x2 Word;
  static constexpr int kWords = 4;  // of a 16-byte unit
  static constexpr short kInfinity = 0x7f80;
  static __device__ __forceinline__ Word of(uint32_t bits) {
    const s16x2 x = __builtin_bit_cast(s16x2, bits);
    return x ^ ((x >> 15) & (short)0x7fff);
  }
  static __device__ __forceinline__ void back(Word w, float (&x)[2]) {
    const uint32_t u = __builtin_bit_cast(uint32_t, of(__builtin_bit_cast(uint32_t, w)));
    x[0] = __uint_as_float(u << 16);
    x[1] = __uint_as_float(u & 0xffff0000u);
  }
  static __device__ __forceinline__ bool finite(Word top, Word low) {
    return max(top[0], top[1]) < kInfinity && min(low[0], low[1]) > (short)~kInfinity;
  }
};
template <>
struct Order<float> {
  typedef int Word;
  static constexpr int kWords = 4;
  static constexpr int kInfinity = 0x7f800000;
  static __device__ __forceinline__ Word of(uint32_t bits) { return (int)bits ^ (((int)bits >> 31) & 0x7fffffff); }
  static __device__ __forceinline__ void back(Word w, float (&x)[1]) { x[0] = __int_as_float(of((uint32_t)w)); }
  static __device__ __forceinline__ bool finite(Word top, Word low) { return top < kInfinity && low > ~kInfinity; }
};

// the lane's words against those of the lanes of its group of four
template <typename W, typename F>
__device__ __forceinline__ W over_four(W x, F f) {
  auto with = [&](auto ctrl) {
    return __builtin_bit_cast(W, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x = f(x, with(std::integral_constant<int, 0xB1>()));     // quad_perm 1 0 3 2
  return f(x, with(std::integral_constant<int, 0x4E>()));  // quad_perm 2 3 0 1
}

template <typename E>
__global__ __launch_bounds__(kSummaryThreads) void kv_summary_kernel(const E* __restrict__ k_cache, int8_t* __restrict__ codes, int8_t* __restrict__ exponents,
                                                                      const int32_t* __restrict__ cu_q, const int32_t* __restrict__ ctx_before,
                                                                      const int32_t* __restrict__ block_table, int bt_stride, int B, int Hkv, int D) {
  constexpr int X = Elem<E>::X, kRounds = 256 / (16 * X);  // rounds of 16 units cover the largest head
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  auto first_unit = [](int cu, int b) { return (cu >> 4) + b; };
  const SeqOf seq = find_sequence(cu_q, ctx_before, B, blockIdx.x, first_unit);
  const int j = (max(seq.cb, 0) >> 4) + (int)blockIdx.x - first_unit(seq.tok0, seq.b);  // (tokens at negative positions fill nothing)
  const int g = blockIdx.y * (kSummaryThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (seq.S <= 0 || j >= (seq.cb + seq.S) >> 4 || g >= Hkv) return;
  const int64_t blk = block_table[(size_t)seq.b * bt_stride + j];
  const E* const src = k_cache + ((size_t)blk * Hkv + g) * 16 * D;
  const int units = D / X, Dp = summary_channels(D);
  typedef Order<E> O;
  typedef typename O::Word Word;
  constexpr int kIn = X / O::kWords;  // keys of a word
  float top[kRounds][X], low[kRounds][X], size = 0.f;
  bool fine = true;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int c = r * 16 + (lane >> 2);
#pragma unroll
    for (int e = 0; e < X; ++e) top[r][e] = low[r][e] = 0.f;
    if (c >= units) continue;
    u4 raw[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) raw[n] = *reinterpret_cast<const u4*>(src + (c * 16 + n * 4 + (lane & 3)) * X);
#pragma unroll
    for (int w = 0; w < O::kWords; ++w) {
      Word most = O::of(raw[0][w]), least = most;
#pragma unroll
      for (int n = 1; n < 4; ++n) {
        const Word x = O::of(raw[n][w]);
        most = __builtin_elementwise_max(most, x);
        least = __builtin_elementwise_min(least, x);
      }
      most = over_four(most, [](Word a, Word b) { return __builtin_elementwise_max(a, b); });
      least = over_four(least, [](Word a, Word b) { return __builtin_elementwise_min(a, b); });
      fine = fine && O::finite(most, least);
      float up[kIn], down[kIn];
      O::back(most, up);
      O::back(least, down);
#pragma unroll
      for (int i = 0; i < kIn; ++i) {
        top[r][w * kIn + i] = up[i];
        low[r][w * kIn + i] = down[i];
        size = fmaxf(size, fmaxf(fabsf(up[i]), fabsf(down[i])));
      }
    }
  }
  fine = __all(fine);
  const int e = code_exponent(wave_max(size));
  int8_t* const to = codes + ((size_t)blk * Hkv + g) * 2 * Dp;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int c = r * 16 + (lane >> 2);
    if (c * X >= Dp || (lane & 3) > 1) continue;
    // lane 0 of the four stores the largest, lane 1 the smallest
    uint32_t out[X / 4];
#pragma unroll
    for (int w = 0; w < X / 4; ++w) {
      out[w] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (so far below the block's largest that fp32 scales it to zero, a key still takes a unit outward)
        const float key = (lane & 1) ? low[r][4 * w + i] : top[r][4 * w + i], scaled = ldexpf(key, -e);
        const float x = (lane & 1) ? (key < 0.f ? fminf(floorf(scaled), -1.f) : floorf(scaled)) : (key > 0.f ? fmaxf(ceilf(scaled), 1.f) : ceilf(scaled));
        out[w] |= (fine ? (uint32_t)(int)x & 0xffu : 0u) << (8 * i);
      }
    }
    uint32_t* const at = reinterpret_cast<uint32_t*>(to + (lane & 1) * Dp + c * X);
    if constexpr (X == 8) *reinterpret_cast<u32x2*>(at) = u32x2{out[0], out[1]};
    else *at = out[0];
  }
  if (lane == 0) exponents[(size_t)blk * Hkv + g] = (int8_t)(fine ? e : kNotFinite);
}

}  // namespace

hipError_t launch_kv_summary(const ecoserve_layout& L, const void* k_cache, void* summary, const int32_t* cu_q, const int32_t* ctx_before,
                             const int32_t* block_table, int32_t bt_stride, int32_t B, int32_t T, hipStream_t s) {
  int8_t* const codes = (int8_t*)summary;
  int8_t* const exponents = codes + summary_code_bytes(L);
  const dim3 grid((unsigned)((int64_t)T / 16 + B), (unsigned)((L.num_kv_heads + 3) / 4));
  if (L.dtype == ECOSERVE_BF16)
    hipLaunchKernelGGL((kv_summary_kernel<uint16_t>), grid, dim3(kSummaryThreads), 0, s, (const uint16_t*)k_cache, codes, exponents, cu_q, ctx_before, block_table,
                       bt_stride, B, L.num_kv_heads, L.head_dim);
  else
    hipLaunchKernelGGL((kv_summary_kernel<float>), grid, dim3(kSummaryThreads), 0, s, (const float*)k_cache, codes, exponents, cu_q, ctx_before, block_table,
                       bt_stride, B, L.num_kv_heads, L.head_dim);
  return hipGetLastError();
}

}  // namespace eco
