// KV-cache append with the position rotation on the way: K and Q rows are turned between the projection and the cache
// (or q_out), V rows are stored as they are.
//
// Pair i of a head vector at position p is turned by theta = p f_i.  theta / 2 pi is a double product, off by three
// roundings of 64 bits at most (3.4e-16 of itself: less than fp32's own rounding up to 2^27 radians, 7e-7 at 2^31); its distance from
// the nearest quarter turn, at most an eighth of a turn, goes to fp32, where the Taylor series of sine and cosine (to a^9 and a^10; the next
// terms are below 2e-9 and 2e-10 there) are as good as the type: no table in memory, whatever the positions.
// The products are fp32, rounded once on the way out.
//
// Memory bounds the large calls (every Q, K and V element is read once and written once), launch latency and three
// round trips the small ones.  An angle serves all heads of a token, so a thread keeps one place of the head vector (16
// bytes, of both halves of the pairs) and one token, has its 4 or 8 angles in registers, and walks the heads.
//
// The blocks of the batch are numbered as in kv_append.hip (cu_q[b] / 16 + 2 b); a workgroup takes the tokens of one
// block and a run of heads of K and Q, or up to four heads of V, whose transposition goes through LDS.
#include <type_traits>

#include "common.h"

namespace eco {

namespace {

constexpr int kRopeThreads = 256;

// What the kernels need of the rotation (by value: the axes of the pairs travel with the launch).
struct Turns {
  const double* inv_freq;
  const int32_t* positions;  // [num_axes][T] or NULL
  int32_t T, rotary, num_axes;
  uint8_t axis[128];
};

struct Angle {
  float c, s;
};
__device__ __forceinline__ Angle angle_of(int32_t position, double inv_freq) {
  const double t = (double)position * (inv_freq * 0.15915494309189535);  // turns
  const double q4 = (t - rint(t)) * 4.0, k = rint(q4);
  const float a = (float)((q4 - k) * 1.5707963267948966), a2 = a * a;
  const float s = a + a * a2 * (-1.f / 6 + a2 * (1.f / 120 + a2 * (-1.f / 5040 + a2 * (1.f / 362880))));
  const float c = 1.f + a2 * (-0.5f + a2 * (1.f / 24 + a2 * (-1.f / 720 + a2 * (1.f / 40320 - a2 * (1.f / 3628800)))));
  const int quarter = (int)k & 3;
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return {quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y};
}
// The angle of pair i of packed token `tok`, at `place` in its sequence.
__device__ __forceinline__ Angle angle_of_pair(const Turns& r, int i, int tok, int place) {
  const int32_t p = r.positions ? r.positions[(size_t)(r.num_axes > 1 ? r.axis[i] : 0) * r.T + tok] : place;
  return angle_of(p, r.inv_freq[i]);
}

template <typename E>
__device__ __forceinline__ float value(E x) {
  return Elem<E>::load(&x);
}
template <typename E>
__device__ __forceinline__ E rounded(float x) {
  E y;
  Elem<E>::store(&y, x);
  return y;
}

// WV elements at a time: a 16-byte unit, or half of one where the halves of the pairs do not begin with a unit.
// kEach (halves, of heads that are not turned as a whole and whose units a wavefront has together): a thread turns one unit and reads the other half of its pairs besides;
// otherwise it turns both.  (Of accesses to the second half few lanes would have any: 32 elements turned, 86 k tokens, 8 heads on 1 of 256 264 us, so 227; 16 k tokens, 64 on 8 of 128
// 173, so 163.  Heads that are turned as a whole: 3 prompts, 3.4 k tokens, 64 on 8 of 128 40.6 us, so 48.6.)  In place the other half's owner has it from memory before either stores: loads
// and stores are instructions of the one wavefront, in this order.
template <typename E, int WV, bool kAdjacent, bool kEach>
__global__ __launch_bounds__(kRopeThreads) void kv_append_rope_kernel(
    E* __restrict__ k_cache, E* __restrict__ v_cache, const E* __restrict__ k_new, const E* __restrict__ v_new, int new_row_stride, const E* q, E* q_out,
    int q_row_stride, int q_out_row_stride, const Turns turns, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ ctx_before,
    const int32_t* __restrict__ block_table, int bt_stride, int B, int Hq, int Hkv, int D, int v_heads, int v_slices, int per_slice) {
  constexpr int X = Elem<E>::X, kAhead = 4;
  struct alignas(WV * sizeof(E)) Unit {
    E e[WV];
  };
  extern __shared__ __attribute__((aligned(16))) char staged[];
  auto first_unit = [](int cu, int b) { return (cu >> 4) + 2 * b; };
  const SeqOf seq = find_sequence(cu_q, ctx_before, B, blockIdx.x, first_unit);
  const int b = seq.b, tok0 = seq.tok0, S = seq.S, cb = seq.cb;
  const int nth = (int)blockIdx.x - first_unit(tok0, b);
  if (S <= 0 || nth > ((cb + S - 1) >> 4) - (cb >> 4)) return;
  const int tid = threadIdx.x, j = (cb >> 4) + nth;
  if (j < 0) return;  // (tokens at negative positions: places of a padded batch)
  const int lo = max(0, cb - (j << 4)), hi = min(16, cb + S - (j << 4));  // addressed slots of the block
  const int t_slot0 = tok0 + (j << 4) - cb;                               // packed token of slot 0 (may lie before tok0)
  const int64_t blk = block_table[(size_t)b * bt_stride + j];

  if ((int)blockIdx.y < v_slices) {
    // V, as in kv_append.hip: rows to LDS, out along the slots
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const int g0 = blockIdx.y * v_heads, heads = min(v_heads, Hkv - g0), upr = D / X, vrow = D + X;
    E* const vt = reinterpret_cast<E*>(staged);
    for (int u = tid; u < heads * 16 * upr; u += kRopeThreads) {
      const int h = u / (16 * upr), r = u % (16 * upr), slot = r / upr, c = r % upr;
      if (slot >= lo && slot < hi)
        *reinterpret_cast<u4*>(vt + ((size_t)h * 16 + slot) * vrow + c * X) =
            *reinterpret_cast<const u4*>(v_new + (size_t)(t_slot0 + slot) * new_row_stride + (g0 + h) * D + c * X);
    }
    __syncthreads();
    E* const vdst = v_cache + ((size_t)blk * Hkv + g0) * D * 16;
    constexpr int kGroups = 16 / X;
    for (int u = tid; u < heads * D * kGroups; u += kRopeThreads) {
      const int row = u / kGroups, s0 = (u % kGroups) * X, h = row / D;  // (row = h D + d)
      const E* const col = vt + (size_t)h * 16 * vrow + (row - h * D);
      E* const dst = vdst + (size_t)row * 16;
      if (s0 >= lo && s0 + X <= hi) {
        alignas(16) E tmp[X];
#pragma unroll
        for (int e = 0; e < X; ++e) tmp[e] = col[(s0 + e) * vrow];
        *reinterpret_cast<u4*>(dst + s0) = *reinterpret_cast<const u4*>(tmp);
      } else {
#pragma unroll
        for (int e = 0; e < X; ++e)
          if (s0 + e >= lo && s0 + e < hi) dst[s0 + e] = col[(s0 + e) * vrow];
      }
    }
    return;
  }

  // K heads, then Q heads: h_begin .. h_end - 1 of the list
  const int R = turns.rotary, half = R >> 1, total = Hkv + (q ? Hq : 0);
  const int h_begin = ((int)blockIdx.y - v_slices) * per_slice, h_end = min(h_begin + per_slice, total);
  const int turned = kAdjacent || kEach ? R / WV : half / WV, places = turned + (D - R) / WV;  // of a head vector, a thread each
  const int per_head = 16 * places, at_once = max(1, kRopeThreads / per_head);
  E* const kdst = k_cache + (size_t)blk * Hkv * 16 * D;
  for (int base = 0; base < per_head; base += kRopeThreads) {
    const int sub = tid / per_head, it = base + tid - sub * per_head, slot = it / places, c = it - slot * places;
    if (sub >= at_once || it >= per_head || slot < lo || slot >= hi) continue;
    const int tok = t_slot0 + slot;
    const bool turn = c < turned, second = kEach && turn && c * WV >= half;  // second: of the second half
    const int e0 = turn ? c * WV : R + (c - turned) * WV;
    constexpr int kPairs = kAdjacent ? WV / 2 : WV;
    Angle an[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) an[i] = Angle{1.f, 0.f};
    if (turn)
#pragma unroll
      for (int i = 0; i < kPairs; ++i) an[i] = angle_of_pair(turns, (second ? c - half / WV : c) * kPairs + i, tok, (j << 4) + slot);
    const E* const krow = k_new + (size_t)tok * new_row_stride + e0;
    const E* const qrow = q + (size_t)tok * q_row_stride + e0;
    E* const orow = q_out + (size_t)tok * q_out_row_stride + e0;
    // where the place lies in a K block of one head; the second half of the pairs
    E* const kplace = kdst + (e0 / X) * 16 * X + slot * X + e0 % X;
    E* const kplace2 = kdst + ((e0 + half) / X) * 16 * X + slot * X + (e0 + half) % X;
    const bool two = !kAdjacent && turn;
    for (int h0 = h_begin + sub; h0 < h_end; h0 += kAhead * at_once) {
      Unit a[kAhead], d[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = min(h0 + n * at_once, h_end - 1);
        const E* const src = h < Hkv ? krow + h * D : qrow + (h - Hkv) * D;
        a[n] = *reinterpret_cast<const Unit*>(src);
        if (two) d[n] = *reinterpret_cast<const Unit*>(second ? src - half : src + half);
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int h = h0 + n * at_once;
        if (h >= h_end) break;
        if (turn) {
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            E& ea = a[n].e[kAdjacent ? 2 * i : i];
            E& eb = kAdjacent ? a[n].e[2 * i + 1] : d[n].e[i];
            const float x = value(ea), y = value(eb);
            ea = rounded<E>(second ? y * an[i].s + x * an[i].c : x * an[i].c - y * an[i].s);
            if (!kEach) eb = rounded<E>(x * an[i].s + y * an[i].c);
          }
        }
        E* const to = h < Hkv ? kplace + (size_t)h * 16 * D : orow + (h - Hkv) * D;
        *reinterpret_cast<Unit*>(to) = a[n];
        if (two && !kEach) *reinterpret_cast<Unit*>(h < Hkv ? kplace2 + (size_t)h * 16 * D : to + half) = d[n];
      }
    }
  }
}

// At most one new token per sequence (the decode step): one wavefront per sequence and up to four heads of K, of V or of Q;
// a lane has the pairs lane and lane + 64 and, of the elements that are not turned, every 64th.
constexpr int kOneHeads = 4;
template <typename E, bool kAdjacent>
__global__ __launch_bounds__(kRopeThreads) void kv_append_rope_one_kernel(
    E* __restrict__ k_cache, E* __restrict__ v_cache, const E* __restrict__ k_new, const E* __restrict__ v_new, int new_row_stride, const E* q, E* q_out,
    int q_row_stride, int q_out_row_stride, const Turns turns, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ ctx_before,
    const int32_t* __restrict__ block_table, int bt_stride, int B, int Hq, int Hkv, int D, int kv_waves, int waves_of_seq) {
  constexpr int X = Elem<E>::X;
  const int wave = blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = wave / waves_of_seq, part = wave - b * waves_of_seq;
  if (b >= B) return;
  const int p = ctx_before[b], tok = cu_q[b], end = cu_q[b + 1];
  if (end - tok <= 0 || p < 0) return;
  const int slot = p & 15;
  if (part < kv_waves) {  // V: element d to [d][slot]
    const int g0 = part * kOneHeads;
    E x[kOneHeads][4];
#pragma unroll
    for (int n = 0; n < kOneHeads; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[n][r] = g0 + n < Hkv && lane + 64 * r < D ? v_new[(size_t)tok * new_row_stride + (g0 + n) * D + lane + 64 * r] : E(0);
    const int64_t blk = block_table[(size_t)b * bt_stride + (p >> 4)];
    E* const vdst = v_cache + ((size_t)blk * Hkv + g0) * D * 16 + slot;
#pragma unroll
    for (int n = 0; n < kOneHeads; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (g0 + n < Hkv && lane + 64 * r < D) vdst[((size_t)n * D + lane + 64 * r) * 16] = x[n][r];
    return;
  }
  const bool is_k = part < 2 * kv_waves;
  const int h0 = (part - (is_k ? kv_waves : 2 * kv_waves)) * kOneHeads, heads = is_k ? Hkv : Hq;
  const E* const src = is_k ? k_new + (size_t)tok * new_row_stride : q + (size_t)tok * q_row_stride;
  const int R = turns.rotary, half = R >> 1;
  E a[kOneHeads][2], d[kOneHeads][2], rest[kOneHeads][4];
  auto first = [&](int i) { return kAdjacent ? 2 * i : i; };
  auto second = [&](int i) { return kAdjacent ? 2 * i + 1 : i + half; };
#pragma unroll
  for (int n = 0; n < kOneHeads; ++n) {
    const E* const row = src + (size_t)min(h0 + n, heads - 1) * D;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int i = lane + 64 * r;
      a[n][r] = i < half ? row[first(i)] : E(0);
      d[n][r] = i < half ? row[second(i)] : E(0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) rest[n][r] = R + lane + 64 * r < D ? row[R + lane + 64 * r] : E(0);
  }
  Angle an[2];
#pragma unroll
  for (int r = 0; r < 2; ++r)
    if (lane + 64 * r < half) an[r] = angle_of_pair(turns, lane + 64 * r, tok, p);
  const int64_t blk = is_k ? block_table[(size_t)b * bt_stride + (p >> 4)] : 0;
  E* const kdst = k_cache + (size_t)blk * Hkv * 16 * D + slot * X;
  E* const qdst = is_k ? nullptr : q_out + (size_t)tok * q_out_row_stride;
  auto put = [&](int h, int e, E x) {
    if (is_k) kdst[(size_t)h * 16 * D + (e / X) * 16 * X + e % X] = x;
    else qdst[(size_t)h * D + e] = x;
  };
#pragma unroll
  for (int n = 0; n < kOneHeads; ++n) {
    if (h0 + n >= heads) break;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int i = lane + 64 * r;
      if (i >= half) continue;
      const float x = value(a[n][r]), y = value(d[n][r]);
      put(h0 + n, first(i), rounded<E>(x * an[r].c - y * an[r].s));
      put(h0 + n, second(i), rounded<E>(x * an[r].s + y * an[r].c));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (R + lane + 64 * r < D) put(h0 + n, R + lane + 64 * r, rest[n][r]);
  }
}

template <typename E, bool kAdjacent>
void launch_typed(const RopeAppend& a, const Turns& turns, int num_cu, hipStream_t s) {
  const int D = a.D;
  E *const kc = (E*)a.k_cache, *const vc = (E*)a.v_cache;
  const E *const kn = (const E*)a.k_new, *const vn = (const E*)a.v_new, *const q = (const E*)a.q;
  E* const qo = (E*)a.q_out;
  if (a.max_new_len <= 1) {
    const int kv_waves = (a.Hkv + kOneHeads - 1) / kOneHeads, of_seq = 2 * kv_waves + (q ? (a.Hq + kOneHeads - 1) / kOneHeads : 0);
    const int64_t waves = (int64_t)a.B * of_seq;
    const int per_wg = waves <= 2 * num_cu ? 1 : kRopeThreads / 64;
    hipLaunchKernelGGL((kv_append_rope_one_kernel<E, kAdjacent>), dim3((unsigned)((waves + per_wg - 1) / per_wg)), dim3(per_wg * 64), 0, s, kc, vc, kn, vn,
                       a.new_row_stride, q, qo, a.q_row_stride, a.q_out_row_stride, turns, a.cu_q, a.ctx_before, a.block_table, a.bt_stride, a.B, a.Hq, a.Hkv, D,
                       kv_waves, of_seq);
    return;
  }
  const int v_heads = D * (int)sizeof(E) <= 512 ? 4 : 2, v_slices = (a.Hkv + v_heads - 1) / v_heads;
  const int64_t units = (int64_t)a.T / 16 + 2 * (int64_t)a.B;
  const int total = a.Hkv + (q ? a.Hq : 0);
  // heads per workgroup: eight workgroups per CU, then more heads to an angle (3 prompts, 3.4 k tokens, 64 heads on 8 of 128, where registers leave four at once: 4 workgroups
  // per CU 43.7 us, 8 40.5, 16 49.0)
  const int64_t want = (8 * (int64_t)num_cu + units - 1) / units;
  const int slices = (int)(want < total ? want : total), per_slice = (total + slices - 1) / slices;
  const dim3 grid((unsigned)units, (unsigned)(v_slices + (total + per_slice - 1) / per_slice));
  const size_t lds = (size_t)v_heads * 16 * (D + Elem<E>::X) * sizeof(E);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), lds, s, kc, vc, kn, vn, a.new_row_stride, q, qo, a.q_row_stride, a.q_out_row_stride, turns, a.cu_q,
                       a.ctx_before, a.block_table, a.bt_stride, a.B, a.Hq, a.Hkv, D, v_heads, v_slices, per_slice);
  };
  constexpr int X = Elem<E>::X;
  if constexpr (kAdjacent) {
    go(&kv_append_rope_kernel<E, X, true, false>);
  } else {
    auto halves = [&](auto units) {
      constexpr int WV = decltype(units)::value;
      if (turns.rotary < D && 64 % (D / WV) == 0) go(&kv_append_rope_kernel<E, WV, false, true>);
      else go(&kv_append_rope_kernel<E, WV, false, false>);
    };
    if (turns.rotary / 2 % X == 0) halves(std::integral_constant<int, X>());
    else halves(std::integral_constant<int, X / 2>());
  }
}

}  // namespace

hipError_t launch_kv_append_rope(const RopeAppend& a, const ecoserve_rope& rope, const double* inv_freq, const int32_t* positions, int num_cu, hipStream_t s) {
  Turns t;
  t.inv_freq = inv_freq;
  t.positions = positions;
  t.T = a.T;
  t.rotary = rope.rotary_dim;
  t.num_axes = rope.num_axes;
  for (int i = 0; i < 128; ++i) t.axis[i] = rope.axis[i];
  const bool adjacent = rope.pairing == ECOSERVE_ROPE_ADJACENT;
  if (a.dtype == ECOSERVE_BF16) adjacent ? launch_typed<uint16_t, true>(a, t, num_cu, s) : launch_typed<uint16_t, false>(a, t, num_cu, s);
  else adjacent ? launch_typed<float, true>(a, t, num_cu, s) : launch_typed<float, false>(a, t, num_cu, s);
  return hipGetLastError();
}

}  // namespace eco
