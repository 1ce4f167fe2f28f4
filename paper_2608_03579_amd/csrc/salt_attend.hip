// Attention over the paged 8-bit cache, for batches whose domains share long prefixes.
//
//   out[t][h] = sum_j p_j v_j,   p = softmax_j(scale q[t][h] . k_j),
//
// j over the token's domain prefix (all of it) and its sequence's own keys up to the
// token's own position; a row without keys gives zeros, a row whose logits are all -inf
// NaN (as the formula does).  The batch is cut into work
// items on the host (salt_seqs.h); a work item runs once per kv head.
//
// One pass over the keys with the running maximum m and sum l of the softmax.  Both
// products run on bf16 matrix instructions with fp32 accumulation: every code of the
// cache is exact in bf16 and its scale multiplies the fp32 logit (k) or probability
// (v), so nothing of the cache is rounded again.  In bf16 contexts q enters as it is and the
// probabilities in two bf16 terms (16 bits: one term's 2^-9 would show beside the
// result's own rounding where a row has few keys); in fp32 contexts both enter in three, 24 bits.
// One term is taken in one place: tiles of more than 16 rows over e4m3, for units that all rows see
// whole (attend_many, which says why): an error of up to 2^-9 of sum p|v| and of out there.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "salt_cache_device.h"
#include "salt_device.h"
#include "salt_layout.h"
#include "salt_seqs.h"
#include "salt_serve.h"

namespace salt {
namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
// Bytes of a 4 x 4 block transposed: word i of the result holds byte i of each input.
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&o)[4]) {
  const uint32_t t0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), t1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), u1 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

// (the instructions themselves: fmaxf first quiets operands that might be signalling NaNs)
__device__ __forceinline__ float max2(float a, float b) {
  return __builtin_amdgcn_fmed3f(a, b, __builtin_inff());
}
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
// What a row's weighted values are multiplied by in the end.  The largest logit above -inf has added about 1 or
// more to the sum l, so l = 0 says that the row has no keys, or (0 / 0) none with a logit above -inf.
__device__ __forceinline__ float inverse_sum(float l, bool has_keys) {
  return l == 0.f ? (has_keys ? __builtin_nanf("") : 0.f) : 1.0f / l;
}
// Whether the rows of the tile's token `ti` have keys.  (asked where their keys are all in this item)
__device__ __forceinline__ bool has_keys(const AttItem& it, int ti) { return it.pre_len > 0 || it.pos0 + ti >= 0; }

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
    const int page = uniform_word(a.pages, ref + (j >> lp));
    // (a uniform base and the lane's own offset)
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    const uint8_t *kb = a.kv.k + vec * D, *vb = a.kv.v + vec * D;
    load_words<D / 16>(kb + lane_offset(r * D + g * (D / 4)), x.k[t]);
    const uint32_t vo = lane_offset(4 * g * D + r * (D / 16));
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words<D / 64>(vb + vo + i * D, x.v[4 * t + i]);
    const float4 s = *reinterpret_cast<const float4*>(a.kv.ks + vec + (uint32_t)(4 * g));
    const float4 u = *reinterpret_cast<const float4*>(a.kv.vs + vec + (uint32_t)(4 * g));
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
  top = row_max(top);
  if (__any(top > w.m + kMaxSlack)) {
    const float m = fmaxf(w.m, top);
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

// A row's result from the lane's part of it (row (l & 15) of a row tile): to out, or as a piece's.
template <typename E, int D>
__device__ __forceinline__ void finish_row(const AttArgs& a, const AttItem& it, int kvh, int row, int g,
                                           const f32x4 (&o)[D / 16], float m, float l) {
  constexpr int DT = D / 16;
  if (row >= it.n_rows) return;
  if (it.out_row < 0) {
    const int ti = row / a.group;
    E* out = reinterpret_cast<E*>(a.out) + (size_t)a.order[it.tok0 + ti] * a.ldo +
             (size_t)(kvh * a.group + row - ti * a.group) * D;
    const float inv = inverse_sum(l, has_keys(it, ti));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; d += 4) {
        const float w0 = o[d][i] * inv, w1 = o[d + 1][i] * inv, w2 = o[d + 2][i] * inv, w3 = o[d + 3][i] * inv;
        E* at = out + (4 * g + i) * DT + d;
        if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(at) = make_float4(w0, w1, w2, w3);
        else *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(w0, w1), pack_bf16x2(w2, w3));
      }
  } else {
    const size_t pr = (size_t)it.out_row + (size_t)kvh * it.n_rows + row;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < DT; d += 4)
        *reinterpret_cast<float4*>(a.part + pr * D + (4 * g + i) * DT + d) =
            make_float4(o[d][i], o[d + 1][i], o[d + 2][i], o[d + 3][i]);
    if (g == 0) *reinterpret_cast<float2*>(a.stat + 2 * pr) = make_float2(m, l);
  }
}

// One item of up to 16 rows, operands straight from memory.  kWaves = 4: the block's waves take 32
// keys in turn, and their results are joined in LDS.  kWaves = 1: one wave alone (the block's others
// have items of their own); no join, and its start-up is paid once for all its keys.  Latency
// bounds small batches (four sequences of up to 1024 keys, 24 heads: 6.2 us, and 4.3 to join), the cache's
// bytes large ones: 64 sequences of 2000 keys, 8 kv heads, 49 us, 5.5 TB/s.
template <int D>
struct FewLds {
  float o[4][16][D + 4];
  float m[4][16], l[4][16];
};
template <typename E, int D, int FMT, int kWaves>
__device__ __forceinline__ void attend_few(const AttArgs& a, const AttItem& it, int kvh, char* lds) {
  using R = Rows<E, D>;
  FewLds<D>& sh = *reinterpret_cast<FewLds<D>*>(lds);
  auto& s_o = sh.o;
  auto& s_m = sh.m;
  auto& s_l = sh.l;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_pre = 2 * ((it.pre_len + kKeyUnit - 1) / kKeyUnit);

  // the first keys are on their way before the rows are looked up
  int st = 2 * it.unit0 + (kWaves == 1 ? 0 : wave);
  const int st1 = 2 * it.unit1;
  Keys<D> x;
  if (st < st1) load_keys<D>(a, it, n_pre, st, kvh, lane, x);
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

  if (st < st1) {
    while (true) {
      const int next = st + kWaves;
      Keys<D> y;
      if (next < st1) load_keys<D>(a, it, n_pre, next, kvh, lane, y);
      use_keys<E, D, FMT>(w, x, c, min_lim);
      if (next >= st1) break;
      x = y;
      st = next;
    }
  }
  const float lw = row_sum(w.l);
  if constexpr (kWaves == 1) {
    finish_row<E, D>(a, it, kvh, r, g, w.o, w.m, lw);
    return;
  }
  // join the waves
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
    const float inv = inverse_sum(l, has_keys(it, rt));
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

// One item of up to 64 RT rows (RT row tiles of 16 to each of four waves), 64 keys at a time: the
// block takes the keys' codes to bf16 once, into LDS in operand order, two buffers, while
// it multiplies the ones before.  Power-of-two scales (e4m3) go into the bf16 values,
// where they are exact; int8's multiply logits and probabilities.  Bound by the vector
// and matrix units in turn: the two waves of a SIMD hardly overlap them.  2048 tokens of 24 heads behind
// two prefixes of 8192 keys: 320 us, 650 TFLOP/s; matrix units busy 33 %, vector units 44 %, the
// rest waits.  The next unit's logits beside this one's exponentials took 380 us: no more of the two
// overlaps.
template <int D>
struct Staged {            // what a lane brings of its wave's 16 keys
  uint32_t k[D / 16];      // key (l & 15): dim / 4 values from dim / 4 (l >> 4) on
  uint32_t v[4][D / 64];   // keys 4 (l >> 4) + i: dim / 16 values from dim / 16 (l & 15) on
  float ks, vs[4];         // their scales
  int last;                // the wave's keys past this one are not there
};

template <typename E, int D, int FMT, int RT>
struct Many {
  static constexpr int NT = sizeof(E) == 4 ? 3 : 1;                        // bf16 terms of q and
  static constexpr int NP = sizeof(E) == 4 ? 3 : 2;                        // of the probabilities
  static constexpr bool kFold = FMT == kKvE4m3;
  static constexpr int KS = D / 32, DT = D / 16;
  static constexpr int kK = 4 * KS * 1024, kBuf = kK + 2 * DT * 1024 + 512;   // a buffer: k, v, 64 scales of each
};

template <typename E, int D, int FMT, int RT>
__device__ __forceinline__ void attend_many(const AttArgs& a, const AttItem& it, int kvh, char* lds) {
  using M = Many<E, D, FMT, RT>;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_pre = (it.pre_len + kKeyUnit - 1) / kKeyUnit;
  const int lp = a.kv.log2_page;

  // a unit's holder: its keys [j0, end), the own ones or the prefix'
  auto unit = [&](int u, int& j0, int& end) {
    const bool own = u >= n_pre;
    j0 = kKeyUnit * (own ? u - n_pre : u);
    end = own ? it.own_end : it.pre_len;
    return own;
  };
  auto fetch = [&](int u, Staged<D>& x) {
    int j0, end;
    const bool own = unit(u, j0, end);
    const int jw = j0 + 16 * wave, j = min(jw, max(end - 1, 0) & ~15);     // (16 keys lie in one page)
    const int page = uniform_word(a.pages, (own ? it.own_ref : it.pre_ref) + (j >> lp));
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    const uint8_t *kb = a.kv.k + vec * D, *vb = a.kv.v + vec * D;
    load_words<D / 16>(kb + lane_offset(r * D + g * (D / 4)), x.k);
    const uint32_t vo = lane_offset(4 * g * D + r * (D / 16));
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words<D / 64>(vb + vo + i * D, x.v[i]);
    x.ks = (a.kv.ks + vec)[(uint32_t)r];
    const float4 s = *reinterpret_cast<const float4*>(a.kv.vs + vec + (uint32_t)(4 * g));
    x.vs[0] = s.x; x.vs[1] = s.y; x.vs[2] = s.z; x.vs[3] = s.w;
    x.last = end - 1 - jw;
  };
  auto put = [&](const Staged<D>& x, char* buf) {
    // k: the wave's subtile, one 16-byte piece per step of 32 values
    const uint32_t nan = x.ks == x.ks ? 0u : 0x7fc07fc0u;
#pragma unroll
    for (int ks = 0; ks < M::KS; ++ks) {
      uint4 w;
      if constexpr (M::kFold) {
        w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.k[2 * ks], x.ks, false));
        w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.k[2 * ks], x.ks, true));
        w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.k[2 * ks + 1], x.ks, false));
        w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.k[2 * ks + 1], x.ks, true));
        w = make_uint4(w.x | nan, w.y | nan, w.z | nan, w.w | nan);
      } else {
        const uint2 lo = codes_bf16<FMT>(x.k[2 * ks]), hi = codes_bf16<FMT>(x.k[2 * ks + 1]);
        w = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
      *reinterpret_cast<uint4*>(buf + ((wave * M::KS + ks) * 64 + lane) * 16) = w;
    }
    // v: four keys of every value, half a piece (the other half is the neighbour wave's)
#pragma unroll
    for (int q = 0; q < D / 64; ++q) {
      uint32_t lo[4], hi[4];               // values 4 q, 4 q + 1 and 4 q + 2, 4 q + 3 of each key
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool gone = 4 * g + i > x.last;
        const uint32_t c = gone ? 0u : x.v[i][q];
        if constexpr (M::kFold) {
          const float s = x.vs[i] == x.vs[i] && !gone ? x.vs[i] : 1.f;
          lo[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, false));
          hi[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, true));
        } else {
          const uint2 w = codes_bf16<FMT>(c);
          lo[i] = w.x;
          hi[i] = w.y;
        }
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t* w = d < 2 ? lo : hi;
        const uint32_t sel = (d & 1) ? 0x07060302u : 0x05040100u;
        *reinterpret_cast<uint2*>(buf + M::kK + (((wave >> 1) * M::DT + 4 * q + d) * 64 + lane) * 16 + (wave & 1) * 8) =
            make_uint2(__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel));
      }
    }
    if constexpr (!M::kFold) {
      float* sc = reinterpret_cast<float*>(buf + M::kBuf - 512) + 16 * wave;
      if (g == 0) sc[r] = x.ks;
      if (r == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[64 + 4 * g + i] = x.vs[i] == x.vs[i] && 4 * g + i <= x.last ? x.vs[i] : 0.f;
      }
    }
  };

  // the first unit is on its way before the rows are looked up
  const int u1 = it.unit1;
  Staged<D> x;
  if (it.unit0 < u1) fetch(it.unit0, x);

  // the wave's rows
  uint4 q[RT][M::NT][M::KS];
  f32x4 o[RT][M::DT], sum[RT];
  float m[RT], l[RT];
  int lim[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = (wave * RT + t) * 16 + r, ti = row / a.group;
    const bool used = row < it.n_rows;
    const int tok = used ? a.order[it.tok0 + ti] : 0;
    const E* p = reinterpret_cast<const E*>(a.q) + (size_t)tok * a.ldq + (size_t)(kvh * a.group + row - ti * a.group) * D +
                 g * (D / 4);
#pragma unroll
    for (int ks = 0; ks < M::KS; ++ks) {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (used) load8(p + 8 * ks, f);
      uint4 tm[M::NT];
      split_terms<M::NT>(f, tm);
#pragma unroll
      for (int n = 0; n < M::NT; ++n) q[t][n][ks] = tm[n];
    }
#pragma unroll
    for (int d = 0; d < M::DT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[t] = kNegInf;
    l[t] = 0.f;
    lim[t] = it.pos0 + ti + 1;
  }
  const int min_lim = it.pos0 + 1;
  const float c = a.scale * kLog2e;

  // s <- the logits (before their scale) of 64 keys and row tiles [T0, T1).
  auto logits = [&](auto first_, auto past_, const char* buf, f32x4(&s)[RT][4]) {
    constexpr int T0 = decltype(first_)::value, T1 = decltype(past_)::value;
    const float* sc = reinterpret_cast<const float*>(buf + M::kBuf - 512);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int t = T0; t < T1; ++t) s[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < M::KS; ++ks) {
        const uint4 k = *reinterpret_cast<const uint4*>(buf + ((kt * M::KS + ks) * 64 + lane) * 16);
#pragma unroll
        for (int t = T0; t < T1; ++t)
#pragma unroll
          for (int n = 0; n < M::NT; ++n) s[t][kt] = mma_bf16(k, q[t][n][ks], s[t][kt]);
      }
      if constexpr (!M::kFold) {
        const float4 k4 = *reinterpret_cast<const float4*>(sc + 16 * kt + 4 * g);
#pragma unroll
        for (int t = T0; t < T1; ++t) {
          s[t][kt][0] *= k4.x; s[t][kt][1] *= k4.y; s[t][kt][2] *= k4.z; s[t][kt][3] *= k4.w;
        }
      }
      if (kt & 1) __builtin_amdgcn_sched_barrier(0);         // (no further ahead: the registers would spill)
    }
  };
  auto largest = [&](const f32x4(&s)[4]) {                   // of a row, in the log2 domain (c > 0)
    float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) top = max3(top, s[e >> 2][e & 3], s[(e + 1) >> 2][(e + 1) & 3]);
    return row_max(max2(top, s[3][3])) * c;
  };
  // The sums, so far relative to the maximum m[t], relative to a larger one.
  auto raise = [&](int t, float top) {
    const float mn = max2(m[t], top);
    const float alpha = mn == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);
    m[t] = mn;
    l[t] *= alpha;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[t][i] *= alpha;
#pragma unroll
    for (int d = 0; d < M::DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[t][d][i] *= alpha;
  };
  // The 64 keys' part of the sums.  NP: bf16 terms of the probabilities.
  auto add = [&](auto np_, auto first_, auto past_, const char* buf, const f32x4(&s)[RT][4]) {
    constexpr int NP = decltype(np_)::value, T0 = decltype(first_)::value, T1 = decltype(past_)::value;
    const float* sc = reinterpret_cast<const float*>(buf + M::kBuf - 512);
    uint4 p[RT][2][NP];
#pragma unroll
    for (int t = T0; t < T1; ++t) {
      const float mu = m[t] == kNegInf ? 0.f : m[t];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(s[t][2 * h + (e >> 2)][e & 3], c, -mu));
        if constexpr (NP > 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) l[t] += x[e];
        }
        if constexpr (!M::kFold) {
          const float4 v0 = *reinterpret_cast<const float4*>(sc + 64 + 32 * h + 4 * g);
          const float4 v1 = *reinterpret_cast<const float4*>(sc + 64 + 32 * h + 16 + 4 * g);
          x[0] *= v0.x; x[1] *= v0.y; x[2] *= v0.z; x[3] *= v0.w;
          x[4] *= v1.x; x[5] *= v1.y; x[6] *= v1.z; x[7] *= v1.w;
        }
        split_terms<NP>(x, p[t][h]);
        if constexpr (NP == 1)
          sum[t] = mma_bf16(make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), p[t][h][0], sum[t]);
      }
      __builtin_amdgcn_sched_barrier(0x100);                 // (reads of LDS may go ahead)
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < M::DT; ++d) {
        const uint4 v = *reinterpret_cast<const uint4*>(buf + M::kK + ((h * M::DT + d) * 64 + lane) * 16);
#pragma unroll
        for (int t = T0; t < T1; ++t)
#pragma unroll
          for (int n = 0; n < NP; ++n) o[t][d] = mma_bf16(v, p[t][h][n], o[t][d]);
        if (d % 8 == 7) __builtin_amdgcn_sched_barrier(0);
      }
  };

  if (it.unit0 < u1) {
    put(x, lds);
    fetch(min(it.unit0 + 1, u1 - 1), x);
    __syncthreads();
    char *cur = lds, *next = lds + M::kBuf;
    int u = it.unit0, j0, end;
    bool own = unit(u, j0, end);
    // (past the end the last unit again, into a buffer that is not read: no branch around it)
    auto stage = [&] {
      put(x, next);                                          // (its readers are behind the last barrier)
      fetch(min(u + 2, u1 - 1), x);
    };
    auto advance = [&] {
      __syncthreads();
      char* const t = cur;
      cur = next;
      next = t;
      own = unit(++u, j0, end);
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, RT> kRT{};
    // a wave without rows only brings its keys
    if (wave * RT * 16 >= it.n_rows)
      while (u < u1) {
        stage();
        advance();
      }
    while (u < u1) {
      // Units that every row sees whole and whose logits pass no row's maximum by much.  e4m3's
      // probabilities enter in one bf16 term here (rows have 64 keys or more); their sum is then
      // of the rounded ones, so that the roundings cancel where a row's weight lies on few
      // keys, and taken as a row of ones in the product, which spares the vector units.
      // A wave that has to raise a maximum leaves the loop (before the unit's barrier) for
      // the general form below: behind a branch in here the sums would be kept twice.
      while (u < u1 && j0 + kKeyUnit <= (own ? min(min_lim, end) : end)) {
        f32x4 s[RT][4];
        logits(k0, kRT, cur, s);
        bool low = false;
#pragma unroll
        for (int t = 0; t < RT; ++t) low |= largest(s[t]) > m[t] + kMaxSlack;
        if (__any(low)) break;
        stage();
        add(std::integral_constant<int, M::kFold && M::NP == 2 ? 1 : M::NP>(), k0, kRT, cur, s);
        advance();
      }
      if (u >= u1) break;
      // Any unit, row tile by row tile (fewer registers).
      stage();
      auto general = [&](auto t_) {
        constexpr int t = decltype(t_)::value;
        constexpr std::integral_constant<int, t + 1> past{};
        f32x4 s[RT][4];
        logits(t_, past, cur, s);
        const int lt = own ? min(lim[t], end) : end;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + 16 * (e >> 2) + 4 * g + (e & 3) >= lt) s[t][e >> 2][e & 3] = kNegInf;
        raise(t, largest(s[t]));
        add(std::integral_constant<int, M::NP>(), t_, past, cur, s);
      };
      general(k0);
      if constexpr (RT == 2) general(std::integral_constant<int, 1>());
      advance();
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)                               // (the row worked out again, not kept over the loop)
    finish_row<E, D>(a, it, kvh, (int)lane_offset((wave * RT + t) * 16 + r), g, o[t], m[t], row_sum(l[t]) + sum[t][0]);
}

// A work item of any kind: the long ones of many rows come first, those of few rows fill the
// places between them.
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256, D <= 128 ? 2 : 1) k_attend(AttArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int n_block = a.n_kind[0] + a.n_kind[1] + a.n_kind[2];   // items that take a block
  int item = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  if (item >= n_block) {
    const int w = (blockIdx.x - n_block * a.kv.kv_heads) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    item = n_block + w / a.kv.kv_heads;
    kvh = w % a.kv.kv_heads;
    if (item >= n_block + a.n_kind[3]) return;
  }
  const AttItem& it = a.items[item];
  if (it.kind == 3) attend_few<E, D, FMT, 1>(a, it, kvh, lds);
  else if (it.kind == 0) attend_few<E, D, FMT, 4>(a, it, kvh, lds);
  else if (it.kind == 1) attend_many<E, D, FMT, 1>(a, it, kvh, lds);
  else if constexpr (attend_rows(sizeof(E), D) == kRowTiles[2]) attend_many<E, D, FMT, 2>(a, it, kvh, lds);
}

// The pieces of a row: 16 lanes per (token, query head).  Lane i reads the maximum and sum of
// pieces i, i + 16, .., so that their weights are known before any of the sums is needed,
// and the sums' reads do not wait for each other.  4.3 us for 96 rows of 8 pieces (three reads
// that wait for one another), 13 us for 49152 rows of 2.
template <typename E, int D>
__global__ void __launch_bounds__(256) k_attend_join(AttArgs a) {
  constexpr int DT = D / 16;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15, d0 = lane * DT;
  if (i >= (int64_t)a.n_joins * a.heads) return;           // (16 lanes leave together)
  const AttJoin j = a.joins[i / a.heads];
  const int h = (int)(i % a.heads), kvh = h / a.group, hr = h - kvh * a.group;
  const int n = j.n[0] + j.n[1];
  auto row_of = [&](int p) {
    const int k = p >= j.n[0];
    return (size_t)(k ? j.row[1] : j.row[0]) +
           (size_t)((k ? p - j.n[0] : p) * a.kv.kv_heads + kvh) * (k ? j.stride[1] : j.stride[0]) +
           (k ? j.r0[1] : j.r0[0]) + hr;
  };
  float m = kNegInf, l = 0.f, v[DT] = {};
  for (int p0 = 0; p0 < n; p0 += 16) {
    // (a piece without keys has the sum 0)
    float2 st = make_float2(kNegInf, 0.f);
    if (p0 + lane < n) st = *reinterpret_cast<const float2*>(a.stat + 2 * row_of(p0 + lane));
    float top = st.x;
#pragma unroll
    for (int x = 1; x < 16; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    const float mn = fmaxf(m, top);
    const float f0 = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    // (a maximum of -inf beside a sum that is not 0: NaN throughout, to be kept)
    const float f1 = st.x == kNegInf ? 1.f : __builtin_amdgcn_exp2f(st.x - mn);
    float ls = st.y * f1;
#pragma unroll
    for (int x = 1; x < 16; x *= 2) ls += __shfl_xor(ls, x);
    l = l * (m == kNegInf && l == 0.f ? 0.f : m == kNegInf ? 1.f : f0) + ls;
#pragma unroll
    for (int d = 0; d < DT; ++d) v[d] *= f0;
    m = mn;
    const int top_p = min(16, n - p0);
    for (int p = 0; p < top_p; p += 4) {                    // (four pieces' reads at a time; past the last one with weight 0)
      float4 x[4][DT / 4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* w = a.part + row_of(p0 + min(p + e, top_p - 1)) * D + d0;
#pragma unroll
        for (int d = 0; d < DT / 4; ++d) x[e][d] = *reinterpret_cast<const float4*>(w + 4 * d);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float w1 = __shfl(f1, min(p + e, 15), 16), f = p + e < top_p ? w1 : 0.f;
        if (f == 0.f) continue;                              // (a sum there may not be finite)
#pragma unroll
        for (int d = 0; d < DT / 4; ++d) {
          v[4 * d] = fmaf(x[e][d].x, f, v[4 * d]); v[4 * d + 1] = fmaf(x[e][d].y, f, v[4 * d + 1]);
          v[4 * d + 2] = fmaf(x[e][d].z, f, v[4 * d + 2]); v[4 * d + 3] = fmaf(x[e][d].w, f, v[4 * d + 3]);
        }
      }
    }
  }
  E* out = reinterpret_cast<E*>(a.out) + (size_t)j.tok * a.ldo + (size_t)h * D + d0;
  const float inv = inverse_sum(l, true);                  // (salt_seqs.h: a joined row has keys)
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
  // (LDS for the kinds that are there)
  const bool many = a.n_kind[1] + a.n_kind[2] > 0;
  const size_t lds = std::max(a.n_kind[0] ? sizeof(FewLds<D>) : 0, many ? 2 * (size_t)Many<E, D, FMT, 1>::kBuf : 0);
  const int blocks = (a.n_kind[0] + a.n_kind[1] + a.n_kind[2]) * a.kv.kv_heads + cdiv(a.n_kind[3] * a.kv.kv_heads, 4);
  hipLaunchKernelGGL((k_attend<E, D, FMT>), dim3(blocks), dim3(256), lds, s, a);
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
