// Norms of the query and key heads with the rotation by position, one pass over q and k.
//
// Of a head x with D values:  v = x / sqrt(mean(x^2) + eps) * w  (v = x without a norm), and of
// its first R values the pairs (a, b) = (v_i, v_{i + R/2}), or (v_2i, v_{2i+1}) interleaved, become
//
//   gain * (a cos t - b sin t,  b cos t + a sin t),   t = position * freq_i,
//
// one rounding at the end.  The angle is taken in revolutions and reduced in 64 bits: at a position of 10^6 an
// fp32 product is off by 0.06 radians.  Reduced to half a revolution it is rounded once (2^-24 of it).
// Bound by memory traffic: 8192 tokens of 32 + 8 heads of 128 in bf16 (168 MB) in 39.4 us on fresh inputs, 4.3 TB/s (a
// large copy: 5.2), and 30.5 where the 84 MB of the inputs come from the Infinity Cache; one token in 3.8 us, a launch
// and two rounds to memory.  (A head's values asked for ahead of the angles: 4.4 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "salt_decode.h"
#include "salt_device.h"
#include "salt_layout.h"

namespace salt {
namespace {

template <typename E, int P>
__device__ __forceinline__ void load_pairs(const E* p, float (&v)[P]) {
  if constexpr (P == 8) {
    Ops<E>::to_f32(Ops<E>::load(p), v);
  } else if constexpr (sizeof(E) == 4) {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = bf_lo(w.x); v[1] = bf_hi(w.x); v[2] = bf_lo(w.y); v[3] = bf_hi(w.y);
  }
}
template <typename E, int P>
__device__ __forceinline__ void store_pairs(E* p, const float (&v)[P]) {
  if constexpr (P == 8) Ops<E>::store(p, v);
  else if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// A wave has one token, and `per` of its heads, query heads first: 64 / L at a time, L lanes to a head, P pairs
// (2 P values) to a lane.  Sines and cosines are worked out once for all of them.  P = 8 reads 16 bytes of bf16 to a
// lane; 4 serves heads and rotated parts that are no multiple of 16.
template <typename E, int P, bool kInter>
__global__ void __launch_bounds__(256) k_rotate(RotateArgs a, int log2_lanes, int per, int slices) {
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = w / slices;
  if (t >= a.T) return;
  const int h0 = (int)(w - t * slices) * per, h1 = min(h0 + per, a.heads + a.kv_heads);
  const int lane = threadIdx.x & 63, lanes = 1 << log2_lanes, step = 64 >> log2_lanes;
  const int p0 = (lane & (lanes - 1)) * P;                 // the lane's first pair
  const bool on = p0 < a.dim / 2, turned = p0 < a.rot / 2;
  // where its values stand: two runs of P (those behind the rotated ones are a run of 2 P)
  const int at0 = kInter || !turned ? 2 * p0 : p0, at1 = kInter || !turned ? 2 * p0 + P : a.rot / 2 + p0;
  float c[P], s[P];
#pragma unroll
  for (int i = 0; i < P; ++i) c[i] = 1.f, s[i] = 0.f;
  if (turned) {
    const double pos = (double)a.pos[t];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const double r = pos * a.freq[p0 + i];
      sincospif(2.f * (float)(r - rint(r)), &s[i], &c[i]);
      s[i] *= a.gain;
      c[i] *= a.gain;
    }
  }
  for (int h = h0 + (lane >> log2_lanes); h < h1; h += step) {   // (the lanes of a head stay together)
    const bool is_q = h < a.heads;
    const int64_t head = (int64_t)(is_q ? h : h - a.heads) * a.dim;
    const E* x = reinterpret_cast<const E*>(is_q ? a.q : a.k) + t * (is_q ? a.ldq : a.ldk) + head;
    float v0[P] = {}, v1[P] = {};
    if (on) {
      load_pairs<E, P>(x + at0, v0);
      load_pairs<E, P>(x + at1, v1);
    }
    const E* g = reinterpret_cast<const E*>(is_q ? a.qw : a.kw);
    if (g) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i) sum = fmaf(v0[i], v0[i], fmaf(v1[i], v1[i], sum));
      for (int m = 1; m < lanes; m *= 2) sum += __shfl_xor(sum, m);
      const float inv = 1.f / sqrtf(sum / (float)a.dim + a.eps);
      float w0[P] = {}, w1[P] = {};
      if (on) {
        load_pairs<E, P>(g + at0, w0);
        load_pairs<E, P>(g + at1, w1);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) v0[i] = v0[i] * inv * w0[i], v1[i] = v1[i] * inv * w1[i];
    }
    float o0[P], o1[P];
    if (kInter && turned) {
      // pair i of the lane: values 2 i and 2 i + 1 of its run
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float u = 2 * i < P ? v0[2 * i % P] : v1[2 * i % P], v = 2 * i < P ? v0[(2 * i + 1) % P] : v1[(2 * i + 1) % P];
        const float ru = u * c[i] - v * s[i], rv = v * c[i] + u * s[i];
        if (2 * i < P) o0[2 * i % P] = ru, o0[(2 * i + 1) % P] = rv;
        else o1[2 * i % P] = ru, o1[(2 * i + 1) % P] = rv;
      }
    } else {
      // (values that are not rotated: by 1 and 0, but for the infinities and NaNs that 0 would spread)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        o0[i] = turned ? v0[i] * c[i] - v1[i] * s[i] : v0[i];
        o1[i] = turned ? v1[i] * c[i] + v0[i] * s[i] : v1[i];
      }
    }
    if (on) {
      E* y = reinterpret_cast<E*>(is_q ? a.qo : a.ko) + t * (is_q ? a.ldqo : a.ldko) + head;
      store_pairs<E, P>(y + at0, o0);
      store_pairs<E, P>(y + at1, o1);
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int bf16, int n_cu, hipStream_t s) {
  const int P = a.dim % 16 == 0 && a.rot % 16 == 0 ? 8 : 4;
  int log2_lanes = 0;
  while ((P << log2_lanes) < a.dim / 2) ++log2_lanes;
  // heads of a wave: as few as it has at a time, or all of a token's where the tokens alone fill the device
  const int step = 64 >> log2_lanes, heads = a.heads + a.kv_heads;
  const int64_t fill = (int64_t)n_cu * 16;
  const int rounds = cdiv(heads, step);
  const int slices = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, fill / std::max(a.T, 1)));
  const int per = cdiv(rounds, slices) * step, n = cdiv(heads, per);
  const dim3 grid((unsigned)(((int64_t)a.T * n + 3) / 4));
  auto go = [&](auto e, auto p) {
    using E = decltype(e);
    constexpr int kP = decltype(p)::value;
    if (a.interleaved) hipLaunchKernelGGL((k_rotate<E, kP, true>), grid, dim3(256), 0, s, a, log2_lanes, per, n);
    else hipLaunchKernelGGL((k_rotate<E, kP, false>), grid, dim3(256), 0, s, a, log2_lanes, per, n);
  };
  auto pairs = [&](auto e) {
    if (P == 8) go(e, std::integral_constant<int, 8>());
    else go(e, std::integral_constant<int, 4>());
  };
  if (bf16) pairs(uint16_t());
  else pairs(float());
  return hipGetLastError();
}

}  // namespace salt
