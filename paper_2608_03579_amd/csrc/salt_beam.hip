// Beam search: the best continuations of each request over its beams and the vocabulary, and the copies of
// cache pages that beams which go on take with them.
//
// A continuation (beam b, token v) is worth  c_b + x_bv,  c_b = score_b - log sum_v exp x_bv.  Within a beam
// the order is that of the logits themselves, so one pass over them finds both what c_b needs and
// the n_out best tokens; the beams meet in 64 bits afterwards, where c_b is added once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "salt_cache_device.h"
#include "salt_decode.h"
#include "salt_layout.h"

namespace salt {
namespace {

// Numbers that order as the values do, 0 below all of them (for -inf, which is no continuation).
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);             // (-0 is 0)
  const uint32_t k = u & 0x80000000u ? ~u : u | 0x80000000u;
  return k <= 0x007fffffu ? 0u : k;                        // (~0xff800000: -inf, and NaNs of that sign)
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// (value, ~token): the larger of two is the better continuation of one beam.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, uint32_t token) { return ((uint64_t)key << 32) | (uint32_t)~token; }

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// The best entries so far, the i-th best in lane i; 0 past the last.
struct Best {
  uint64_t e = 0;
  // `v` (the same in all lanes) goes to its place; the entries behind move up a lane.
  __device__ __forceinline__ void insert(uint64_t v) {
    const int at = __popcll(__ballot(e > v));
    const uint64_t up = __shfl_up(e, 1);
    const int lane = threadIdx.x & 63;
    e = lane < at ? e : lane == at ? v : up;
  }
};

// One piece of one row: a block of four waves, which take runs of 512 logits in turn.
template <typename E>
__global__ void __launch_bounds__(256) k_beam_scan(BeamArgs a) {
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.n_out;
  const int chunks = (a.vocab + 511) / 512;
  const int c0 = (int)((int64_t)chunks * split / a.splits), c1 = (int)((int64_t)chunks * (split + 1) / a.splits);
  const E* x = reinterpret_cast<const E*>(a.logits) + (int64_t)row * a.ld;
  Best best;
  uint32_t least = 0;                                      // what a logit has to be above: key of the n-th best
  float m = kNegInf;
  double sum = 0.;
  auto load = [&](int c, float (&v)[8]) {
    const int at = c * 512 + lane * 8;
    if (at + 8 <= a.vocab) {
      load8(x + at, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f[1] = {kNegInf};
        if (at + i < a.vocab) {
          if constexpr (sizeof(E) == 4) f[0] = x[at + i];
          else f[0] = __uint_as_float((uint32_t)x[at + i] << 16);
        }
        v[i] = f[0];
      }
    }
  };
  float v[8], next[8];
  int c = c0 + wave;
  if (c < c1) load(c, v);
  while (c < c1) {
    if (c + 4 < c1) load(c + 4, next);
    // the sum of exponentials under the lane's own maximum
    const float top = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    if (top > m) {
      if (m > kNegInf) sum *= (double)__builtin_amdgcn_exp2f((m - top) * kLog2e);
      m = top;
    }
    const float mu = m == kNegInf ? 0.f : m;
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) part += __builtin_amdgcn_exp2f((v[i] - mu) * kLog2e);
    sum += (double)part;
    uint64_t who = __ballot(order_of(top) > least);        // (NaNs: the row offers nothing in the end)
    while (who) {
      const int from = __builtin_ctzll(who);
      who &= who - 1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t key = order_of(__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[i]), from)));
        if (key <= least) continue;                        // (equal: the ones before have lower tokens)
        best.insert(entry_of(key, (uint32_t)(c * 512 + from * 8 + i)));
        least = (uint32_t)(lane_value(best.e, n - 1) >> 32);
      }
    }
    c += 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = next[i];
  }
  // the waves' lists: an entry's place is the number of better ones
  __shared__ uint64_t list[4 * kMaxOut];
  __shared__ float s_m[4];
  __shared__ double s_sum[4];
  if (lane < n) list[wave * n + lane] = best.e;
  float mw = m;
  for (int i = 1; i < 64; i *= 2) mw = fmaxf(mw, __shfl_xor(mw, i));
  if (m > kNegInf) sum *= (double)__builtin_amdgcn_exp2f((m - mw) * kLog2e);
  for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
  if (lane == 0) s_m[wave] = mw, s_sum[wave] = sum;
  __syncthreads();
  const int64_t piece = (int64_t)row * a.splits + split;
  if (threadIdx.x < 4 * n) {
    const uint64_t e = list[threadIdx.x];
    int at = 0;
    for (int i = 0; i < 4 * n; ++i) at += list[i] > e || (list[i] == e && i < (int)threadIdx.x);
    if (at < n) a.best[piece * n + at] = e;
  }
  if (threadIdx.x == 0) {
    const float mm = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    double t = 0.;
    for (int i = 0; i < 4; ++i)
      t += s_m[i] > kNegInf ? s_sum[i] * (double)__builtin_amdgcn_exp2f((s_m[i] - mm) * kLog2e) : s_sum[i];
    a.stat[piece] = make_double2((double)mm, t);
  }
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  for (int i = 1; i < 64; i *= 2) {
    const uint64_t o = __shfl_xor(v, i);
    v = o > v ? o : v;
  }
  return v;
}

// One request: the pieces of each beam joined, then the beams.
__global__ void __launch_bounds__(256) k_beam_join(BeamArgs a) {
  const int req = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n_out;
  __shared__ uint64_t list[kMaxBeams * kMaxOut];
  __shared__ double s_c[kMaxBeams];
  for (int b = wave; b < a.width; b += 4) {
    const int64_t row = (int64_t)req * a.width + b, piece = row * a.splits + lane;
    double2 st = make_double2(-__builtin_inf(), 0.);
    if (lane < a.splits) st = a.stat[piece];
    double m = st.x;
    for (int i = 1; i < 64; i *= 2) m = fmax(m, __shfl_xor(m, i));
    double sum = st.x > -__builtin_inf() ? st.y * exp(st.x - m) : st.y;
    for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
    // (a row with a NaN or +inf has a sum of NaN, one without a logit above -inf a sum of 0)
    const float score = a.score[row];
    const bool live = score > kNegInf && score < __builtin_inff() && sum > 0.;
    if (lane == 0) s_c[b] = (double)score - (m + log(sum));
    // the best of the heads of the pieces' lists, n times
    int next = 1;
    uint64_t head = live && lane < a.splits ? a.best[piece * n] : 0;
    for (int i = 0; i < n; ++i) {
      const uint64_t top = wave_max(head);
      if (lane == 0) list[b * n + i] = top;
      if (top && head == top) head = next < n ? a.best[piece * n + next++] : 0;
    }
  }
  __syncthreads();
  if (wave) return;
  int next = 1;
  uint64_t head = lane < a.width ? list[lane * n] : 0;
  const double c = lane < a.width ? s_c[lane] : 0.;
  for (int i = 0; i < n; ++i) {
    const double none = -__builtin_inf();
    double top = head ? (double)value_of((uint32_t)(head >> 32)) + c : none;
    const double mine = top;
    for (int k = 1; k < 64; k *= 2) top = fmax(top, __shfl_xor(top, k));
    const uint64_t who = __ballot(head && mine == top);    // (ties: the lowest beam)
    const int from = who ? __builtin_ctzll(who) : 0;
    if (lane == from) {
      const int64_t at = (int64_t)req * n + i;
      a.out_score[at] = who ? (float)top : kNegInf;
      a.out_beam[at] = who ? from : -1;
      a.out_token[at] = who ? (int32_t)~(uint32_t)head : -1;
      if (who) head = next < n ? list[lane * n + next++] : 0;
    }
  }
}

// A block takes one kv head of one page in one layer.
__global__ void __launch_bounds__(256) k_copy_pages(CopyArgs a) {
  const int pair = blockIdx.x / a.kv.kv_heads, h = blockIdx.x % a.kv.kv_heads, layer = blockIdx.y;
  const int lp = a.kv.log2_page, n = a.tokens[pair];
  const size_t from = ((size_t)a.src[pair] * a.kv.kv_heads + h) << lp, to = ((size_t)a.dst[pair] * a.kv.kv_heads + h) << lp;
  const size_t off = a.layer * layer;
  const int vecs = n * a.kv.dim / 16;
  const uint4 *k0 = reinterpret_cast<const uint4*>(a.kv.k + off + from * a.kv.dim),
              *v0 = reinterpret_cast<const uint4*>(a.kv.v + off + from * a.kv.dim);
  uint4 *k1 = reinterpret_cast<uint4*>(a.kv.k + off + to * a.kv.dim), *v1 = reinterpret_cast<uint4*>(a.kv.v + off + to * a.kv.dim);
  for (int i = threadIdx.x; i < vecs; i += 256) {
    const uint4 k = k0[i], v = v0[i];
    k1[i] = k;
    v1[i] = v;
  }
  auto at = [&](void* p, size_t o) { return reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(p) + o); };
  for (int i = threadIdx.x; i < n; i += 256) {
    at(a.kv.ks, off)[to + i] = at(a.kv.ks, off)[from + i];
    at(a.kv.vs, off)[to + i] = at(a.kv.vs, off)[from + i];
    if (a.kv.weight) {
      const size_t mo = a.mark_layer * layer;
      at(a.kv.weight, mo)[to + i] = at(a.kv.weight, mo)[from + i];
      at(a.kv.place, mo)[to + i] = at(a.kv.place, mo)[from + i];
    }
  }
}

}  // namespace

hipError_t launch_beam(const BeamArgs& a, int bf16, hipStream_t s) {
  const dim3 grid(a.splits * a.reqs * a.width);
  if (bf16) hipLaunchKernelGGL(k_beam_scan<uint16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_beam_scan<float>, grid, dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_beam_join, dim3(a.reqs), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_copy_pages, dim3(a.n * a.kv.kv_heads, a.n_layers), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace salt
