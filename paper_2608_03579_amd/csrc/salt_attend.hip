// Attention over the paged 8-bit cache, for batches whose domains share long prefixes.
//
//   out[t][h] = sum_j p_j v_j,   p = softmax_j(scale q[t][h] . k_j),
//
// j over the token's domain prefix (all of it) and its sequence's own keys up to the
// token's own position; a row without keys gives zeros.  The batch is cut into work
// items on the host (salt_seqs.h); a work item runs once per kv head.
//
// One pass over the keys with the running maximum m and sum l of the softmax.  Both
// products run on bf16 matrix instructions with fp32 accumulation: every code of the
// cache is exact in bf16 and its scale multiplies the fp32 logit (k) or probability
// (v), so nothing of the cache is rounded again.  In bf16 contexts q enters as it is and the
// probabilities in two bf16 terms (16 bits: one term's 2^-8 would show beside the
// result's own rounding where a row has few keys); in fp32 contexts both enter in three, 24 bits.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "salt_device.h"
#include "salt_layout.h"
#include "salt_seqs.h"
#include "salt_serve.h"

namespace salt {
namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ f32x4 mma_bf16(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// Four codes (a word) as bf16, in order.
template <int FMT>
__device__ __forceinline__ uint2 codes_bf16(uint32_t w) {
  if constexpr (FMT == kKvInt8) {
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = (float)((int)(w << (24 - 8 * e)) >> 24);
    return make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
  } else {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
  }
}

// Bytes of a 4 x 4 block transposed: word i of the result holds byte i of each input.
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&o)[4]) {
  const uint32_t t0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), t1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), u1 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

template <int N>   // words
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const uint4 a = *reinterpret_cast<const uint4*>(p + 4 * j);
      w[j] = a.x; w[j + 1] = a.y; w[j + 2] = a.z; w[j + 3] = a.w;
    }
  }
}

// x[8] as NT bf16 terms whose sum is x (NT = 1: rounded).
template <int NT>
__device__ __forceinline__ void split_terms(const float (&x)[8], uint4 (&o)[NT]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    o[n] = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
    if (n + 1 < NT) {
      float b[8];
      Ops<uint16_t>::to_f32(o[n], b);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] -= b[e];
    }
  }
}

// The widest of a lane's four: lanes l, l ^ 16, l ^ 32, l ^ 48 hold one row.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// What a lane holds of 32 keys: k of keys (l & 15) and 16 + (l & 15), dim / 4 values
// each from dim / 4 (l >> 4) on; v of keys 4 (l >> 4) .. + 3 and 16 + those, dim / 16
// values each from dim / 16 (l & 15) on; and those eight keys' scales.
template <int D>
struct Keys {
  uint32_t k[2][D / 16];
  uint32_t v[8][D / 64];
  float ks[8], vs[8];
  int end;                 // keys of the holder (j0 + key < end is a key)
  int j0;                  // first key
  bool own;
};

template <int D>
__device__ __forceinline__ void load_keys(const AttArgs& a, const AttItem& it, int n_pre, int step, int kvh, int lane,
                                          Keys<D>& x) {
  // (uniform over the wave)
  x.own = step >= n_pre;
  x.j0 = 32 * (x.own ? step - n_pre : step);
  x.end = x.own ? it.own_end : it.pre_len;
  const int ref = x.own ? it.own_ref : it.pre_ref, last = max(x.end - 1, 0);
  const int lp = a.kv.log2_page, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int j = min(x.j0 + 16 * t, last & ~15);         // a run of 16 keys lies in one page
    const int page = a.pages[ref + (j >> lp)];
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    load_words<D / 16>(a.kv.k + vec * D + r * D + g * (D / 4), x.k[t]);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words<D / 64>(a.kv.v + vec * D + (4 * g + i) * D + r * (D / 16), x.v[4 * t + i]);
    const float4 s = *reinterpret_cast<const float4*>(a.kv.ks + vec + 4 * g);
    const float4 u = *reinterpret_cast<const float4*>(a.kv.vs + vec + 4 * g);
    x.ks[4 * t] = s.x; x.ks[4 * t + 1] = s.y; x.ks[4 * t + 2] = s.z; x.ks[4 * t + 3] = s.w;
    x.vs[4 * t] = u.x; x.vs[4 * t + 1] = u.y; x.vs[4 * t + 2] = u.z; x.vs[4 * t + 3] = u.w;
  }
}

// The running softmax of up to 16 rows, and one wave's part of its keys.
template <typename E, int D>
struct Rows {
  static constexpr int NT = sizeof(E) == 4 ? 3 : 1, NP = sizeof(E) == 4 ? 3 : 2;   // bf16 terms of q, of p
  static constexpr int KS = D / 32, DT = D / 16;
  uint4 q[NT][KS];         // row (l & 15), values of the lane's k
  f32x4 o[DT];             // row (l & 15): values DT (4 (l >> 4) + i) + dt of v's sum
  float m, l;              // maximum (log2 domain) of the row, sum of this lane's keys
  int lim;                 // own keys the row sees
};

template <typename E, int D, int FMT>
__device__ __forceinline__ void use_keys(Rows<E, D>& w, Keys<D>& x, float c, int min_lim) {
  using R = Rows<E, D>;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  f32x4 s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      const uint2 lo = codes_bf16<FMT>(x.k[t][2 * ks]), hi = codes_bf16<FMT>(x.k[t][2 * ks + 1]);
      const uint4 k = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
      for (int n = 0; n < R::NT; ++n) s[t] = mma_bf16(k, w.q[n][ks], s[t]);
    }
  }
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = s[e >> 2][e & 3] * (x.ks[e] * c);
  // keys some row does not see, or that are not there
  const bool edge = x.j0 + 32 > (x.own ? min_lim : x.end);
  const int lim = x.own ? min(w.lim, x.end) : x.end;
  if (edge) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = x.j0 + 16 * (e >> 2) + 4 * g + (e & 3);
      if (j >= lim) y[e] = kNegInf;
      if (j >= x.end) {                      // whatever the page holds there
        x.vs[e] = 0.f;
#pragma unroll
        for (int q = 0; q < D / 64; ++q) x.v[e][q] = 0u;
      }
    }
  }
  float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
  const float m = fmaxf(w.m, row_max(top));
  if (__any(m > w.m)) {
    const float alpha = m == kNegInf ? 1.f : __builtin_amdgcn_exp2f(w.m - m);
    w.l *= alpha;
#pragma unroll
    for (int d = 0; d < R::DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) w.o[d][i] *= alpha;
    w.m = m;
  }
  const float mu = w.m == kNegInf ? 0.f : w.m;
  float p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = __builtin_amdgcn_exp2f(y[e] - mu);
    w.l += p[e];
    // (a v that is not finite made its k's scale NaN; its own must not reach rows that do not see it)
    p[e] *= x.vs[e] == x.vs[e] ? x.vs[e] : 0.f;
  }
  uint4 pt[R::NP];
  split_terms<R::NP>(p, pt);
#pragma unroll
  for (int q = 0; q < D / 64; ++q) {
    uint32_t a[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t in[4] = {x.v[4 * t][q], x.v[4 * t + 1][q], x.v[4 * t + 2][q], x.v[4 * t + 3][q]};
      transpose4(in, a[t]);
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint2 lo = codes_bf16<FMT>(a[0][d]), hi = codes_bf16<FMT>(a[1][d]);
      const uint4 v = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
      for (int n = 0; n < R::NP; ++n) w.o[4 * q + d] = mma_bf16(v, pt[n], w.o[4 * q + d]);
    }
  }
}

template <typename E>
__device__ __forceinline__ void load8(const E* p, float (&v)[8]) { Ops<E>::to_f32(Ops<E>::load(p), v); }

// One item of up to 16 rows: the block's four waves take 32 keys in turn, and their
// results are joined in LDS.
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256) k_attend_few(AttArgs a) {
  using R = Rows<E, D>;
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float s_o[4][16][LD];
  __shared__ float s_m[4][16], s_l[4][16];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.kv.kv_heads;
  const AttItem& it = a.items[blockIdx.x / a.kv.kv_heads];
  const int n_pre = 2 * ((it.pre_len + kKeyUnit - 1) / kKeyUnit);

  R w;
  const int ti = r / a.group;
  {
    const bool used = r < it.n_rows;
    const int tok = used ? a.order[it.tok0 + ti] : 0;
    const E* q = reinterpret_cast<const E*>(a.q) + (size_t)tok * a.ldq + (size_t)(kvh * a.group + r - ti * a.group) * D +
                 g * (D / 4);
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (used) load8(q + 8 * ks, f);
      uint4 tm[R::NT];
      split_terms<R::NT>(f, tm);
#pragma unroll
      for (int n = 0; n < R::NT; ++n) w.q[n][ks] = tm[n];
    }
  }
#pragma unroll
  for (int d = 0; d < R::DT; ++d) w.o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  w.m = kNegInf;
  w.l = 0.f;
  w.lim = it.pos0 + ti + 1;
  const int min_lim = it.pos0 + 1;
  const float c = a.scale * kLog2e;

  int st = 2 * it.unit0 + wave;
  const int st1 = 2 * it.unit1;
  if (st < st1) {
    Keys<D> x;
    load_keys<D>(a, it, n_pre, st, kvh, lane, x);
    while (true) {
      const int next = st + 4;
      Keys<D> y;
      if (next < st1) load_keys<D>(a, it, n_pre, next, kvh, lane, y);
      use_keys<E, D, FMT>(w, x, c, min_lim);
      if (next >= st1) break;
      x = y;
      st = next;
    }
  }
  // join the waves
  const float lw = row_sum(w.l);
  if (g == 0) {
    s_m[wave][r] = w.m;
    s_l[wave][r] = lw;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < R::DT; d += 4)
      *reinterpret_cast<float4*>(&s_o[wave][r][(4 * g + i) * R::DT + d]) =
          make_float4(w.o[d][i], w.o[d + 1][i], w.o[d + 2][i], w.o[d + 3][i]);
  __syncthreads();
  const int row = tid >> 4, d0 = (tid & 15) * R::DT;
  if (row >= it.n_rows) return;
  const float m = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
  float l = 0.f, v[R::DT] = {};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float f = s_m[q][row] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(s_m[q][row] - m);
    if (s_m[q][row] == kNegInf && s_l[q][row] == 0.f) continue;      // no key of this wave's
    l += f * s_l[q][row];
#pragma unroll
    for (int d = 0; d < R::DT; ++d) v[d] += f * s_o[q][row][d0 + d];
  }
  if (it.out_row < 0) {
    const int rt = row / a.group;
    E* out = reinterpret_cast<E*>(a.out) + (size_t)a.order[it.tok0 + rt] * a.ldo +
             (size_t)(kvh * a.group + row - rt * a.group) * D + d0;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < R::DT; d += 4) {
      if constexpr (sizeof(E) == 4)
        *reinterpret_cast<float4*>(out + d) = make_float4(v[d] * inv, v[d + 1] * inv, v[d + 2] * inv, v[d + 3] * inv);
      else
        *reinterpret_cast<uint2*>(out + d) = make_uint2(pack_bf16x2(v[d] * inv, v[d + 1] * inv),
                                                        pack_bf16x2(v[d + 2] * inv, v[d + 3] * inv));
    }
    return;
  }
  const size_t pr = (size_t)it.out_row + (size_t)kvh * it.n_rows + row;
#pragma unroll
  for (int d = 0; d < R::DT; d += 4)
    *reinterpret_cast<float4*>(a.part + pr * D + d0 + d) = make_float4(v[d], v[d + 1], v[d + 2], v[d + 3]);
  if ((tid & 15) == 0) *reinterpret_cast<float2*>(a.stat + 2 * pr) = make_float2(m, l);
}

// The pieces of a row: 16 lanes per (token, query head).
template <typename E, int D>
__global__ void __launch_bounds__(256) k_attend_join(AttArgs a) {
  constexpr int DT = D / 16;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int d0 = (threadIdx.x & 15) * DT;
  if (i >= (int64_t)a.n_joins * a.heads) return;
  const AttJoin& j = a.joins[i / a.heads];
  const int h = (int)(i % a.heads), kvh = h / a.group, hr = h - kvh * a.group;
  float m = kNegInf, l = 0.f, v[DT] = {};
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int p = 0; p < j.n[k]; ++p) {
      const size_t pr = (size_t)j.row[k] + (size_t)(p * a.kv.kv_heads + kvh) * j.stride[k] + j.r0[k] + hr;
      const float2 s = *reinterpret_cast<const float2*>(a.stat + 2 * pr);
      float w[DT];
#pragma unroll
      for (int d = 0; d < DT; d += 4) {
        const float4 x = *reinterpret_cast<const float4*>(a.part + pr * D + d0 + d);
        w[d] = x.x; w[d + 1] = x.y; w[d + 2] = x.z; w[d + 3] = x.w;
      }
      if (s.x == kNegInf && s.y == 0.f) continue;           // no key in this piece
      const float mn = fmaxf(m, s.x);
      const float f0 = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      const float f1 = s.x == kNegInf ? 1.f : __builtin_amdgcn_exp2f(s.x - mn);
      l = l * f0 + s.y * f1;
#pragma unroll
      for (int d = 0; d < DT; ++d) v[d] = v[d] * f0 + w[d] * f1;
      m = mn;
    }
  E* out = reinterpret_cast<E*>(a.out) + (size_t)j.tok * a.ldo + (size_t)h * D + d0;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int d = 0; d < DT; d += 4) {
    if constexpr (sizeof(E) == 4)
      *reinterpret_cast<float4*>(out + d) = make_float4(v[d] * inv, v[d + 1] * inv, v[d + 2] * inv, v[d + 3] * inv);
    else
      *reinterpret_cast<uint2*>(out + d) = make_uint2(pack_bf16x2(v[d] * inv, v[d + 1] * inv),
                                                      pack_bf16x2(v[d + 2] * inv, v[d + 3] * inv));
  }
}

template <typename E, int D, int FMT>
void launch_typed(const AttArgs& a, hipStream_t s) {
  if (a.n_kind[0])
    hipLaunchKernelGGL((k_attend_few<E, D, FMT>), dim3(a.n_kind[0] * a.kv.kv_heads), dim3(256), 0, s, a);
  if (a.n_joins)
    hipLaunchKernelGGL((k_attend_join<E, D>), dim3((unsigned)(((int64_t)a.n_joins * a.heads + 15) / 16)), dim3(256), 0,
                       s, a);
}
template <typename E, int D>
void launch_format(const AttArgs& a, hipStream_t s) {
  if (a.kv.format == kKvInt8) launch_typed<E, D, kKvInt8>(a, s);
  else launch_typed<E, D, kKvE4m3>(a, s);
}
template <typename E>
void launch_dim(const AttArgs& a, hipStream_t s) {
  if (a.kv.dim == 64) launch_format<E, 64>(a, s);
  else if (a.kv.dim == 128) launch_format<E, 128>(a, s);
  else launch_format<E, 256>(a, s);
}

}  // namespace

hipError_t launch_attend(const AttArgs& a, int bf16, hipStream_t s) {
  if (bf16) launch_dim<uint16_t>(a, s);
  else launch_dim<float>(a, s);
  return hipGetLastError();
}

}  // namespace salt
