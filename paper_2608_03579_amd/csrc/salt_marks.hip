// Marks of a tracked cache: the attention weight that each cached token has gathered, and its position; and the
// eviction that goes by them.
//
// The weight that a step adds to token j of a sequence, for each kv head:
//
//   w_j = sum_t sum_h softmax_i(scale q[t][h] . k_i)[j],
//
// t over the step's counted tokens that see j, h over the query heads of the kv head, i over all keys that
// the attention of t reads (prefix and own).  Two passes over the keys: the first finds the maximum and sum of
// every row (k_score_stat, over the attention's own work items; k_score_join where a row is in pieces),
// the second goes by keys and adds up exp2(logit - maximum) / sum over the rows (k_score_add): every
// mark has one owner and is written once, so no atomics, and the sum's order is fixed.
// Codes are exact in bf16; q enters as it is in bf16 contexts, in three bf16 terms (24 bits) in fp32 ones.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "salt_cache_device.h"
#include "salt_decode.h"
#include "salt_layout.h"

namespace salt {
namespace {

template <typename E>
constexpr int terms() { return sizeof(E) == 4 ? 3 : 1; }   // bf16 terms of q

// A query row's values that one lane brings to the products: from dim / 4 g on.
template <typename E, int D>
__device__ __forceinline__ void load_query(const E* q, bool used, uint4 (&o)[terms<E>()][D / 32]) {
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    if constexpr (sizeof(E) == 2) {
      o[0][ks] = used ? *reinterpret_cast<const uint4*>(q + 8 * ks) : make_uint4(0u, 0u, 0u, 0u);
    } else {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (used) load8(q + 8 * ks, f);
      uint4 t[terms<E>()];
      split_terms<terms<E>()>(f, t);
#pragma unroll
      for (int n = 0; n < terms<E>(); ++n) o[n][ks] = t[n];
    }
  }
}

// Logits of 16 keys (the lane: keys 4 g + i) and 16 rows (row l & 15), times 1.
template <typename E, int D, int FMT>
__device__ __forceinline__ f32x4 logits16(const uint32_t (&k)[D / 16], const uint4 (&q)[terms<E>()][D / 32]) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    const uint2 lo = codes_bf16<FMT>(k[2 * ks]), hi = codes_bf16<FMT>(k[2 * ks + 1]);
    const uint4 kb = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
    for (int n = 0; n < terms<E>(); ++n) s = mma_bf16(kb, q[n][ks], s);
  }
  return s;
}

// 32 keys of an item: as the attention has them, without v.
template <int D>
struct Keys32 {
  uint32_t k[2][D / 16];
  float ks[8];
  int end, j0;
  bool own;
};
template <int D>
__device__ __forceinline__ void load_keys32(const AttArgs& a, const AttItem& it, int n_pre, int step, int kvh, int lane,
                                            Keys32<D>& x) {
  x.own = step >= n_pre;
  x.j0 = 32 * (x.own ? step - n_pre : step);
  x.end = x.own ? it.own_end : it.pre_len;
  const int ref = x.own ? it.own_ref : it.pre_ref, last = max(x.end - 1, 0);
  const int lp = a.kv.log2_page, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int j = min(x.j0 + 16 * t, last & ~15);         // a run of 16 keys lies in one page
    const int page = uniform_word(a.pages, ref + (j >> lp));
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    load_words<D / 16>(a.kv.k + vec * D + lane_offset(r * D + g * (D / 4)), x.k[t]);
    const float4 s = *reinterpret_cast<const float4*>(a.kv.ks + vec + (uint32_t)(4 * g));
    x.ks[4 * t] = s.x; x.ks[4 * t + 1] = s.y; x.ks[4 * t + 2] = s.z; x.ks[4 * t + 3] = s.w;
  }
}

// What a row's exponentials are multiplied by: 1 / sum.  A sum of 0: no key has a logit above -inf, and the
// weights are NaN, as the formula's.
__device__ __forceinline__ float2 row_final(float m, float l) {
  return make_float2(m == kNegInf ? 0.f : m, l == 0.f ? __builtin_nanf("") : 1.0f / l);
}

// One item: kWaves = 4: 16 rows, the block's waves take 32 keys in turn; 1: one wave alone.
// RT > 0 instead: 64 RT rows, 16 RT to a wave, which reads all the item's keys.
template <typename E, int D, int FMT, int kWaves, int RT>
__device__ __forceinline__ void stat_item(const ScoreArgs& sa, const AttItem& it, int kvh, float* lds) {
  const AttArgs& a = sa.att;
  constexpr int NR = RT > 0 ? RT : 1;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = kWaves == 1 && RT == 0 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_pre = 2 * ((it.pre_len + kKeyUnit - 1) / kKeyUnit);
  const int row0 = RT > 0 ? wave * 16 * RT : 0;
  if (RT > 0 && row0 >= it.n_rows) return;
  int st = 2 * it.unit0 + (RT > 0 || kWaves == 1 ? 0 : wave);
  const int st1 = 2 * it.unit1, by = RT > 0 ? 1 : kWaves;
  Keys32<D> x;
  if (st < st1) load_keys32<D>(a, it, n_pre, st, kvh, lane, x);
  uint4 q[NR][terms<E>()][D / 32];
  float m[NR], l[NR];
  int lim[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int row = row0 + 16 * t + r, ti = row / a.group;
    const bool used = row < it.n_rows;
    const int tok = used ? a.order[it.tok0 + ti] : 0;
    load_query<E, D>(reinterpret_cast<const E*>(a.q) + (size_t)tok * a.ldq + (size_t)(kvh * a.group + row - ti * a.group) * D +
                         g * (D / 4), used, q[t]);
    m[t] = kNegInf;
    l[t] = 0.f;
    lim[t] = it.pos0 + ti + 1;
  }
  const int min_lim = it.pos0 + row0 / a.group + 1;
  const float c = a.scale * kLog2e;
  while (st < st1) {
    const int next = st + by;
    Keys32<D> y;
    if (next < st1) load_keys32<D>(a, it, n_pre, next, kvh, lane, y);
    const bool edge = x.j0 + 32 > (x.own ? min_lim : x.end);
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      float z[8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x4 s = logits16<E, D, FMT>(x.k[u], q[t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[4 * u + e] = s[e] * (x.ks[4 * u + e] * c);
      }
      if (edge) {
        const int lt = x.own ? min(lim[t], x.end) : x.end;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (x.j0 + 16 * (e >> 2) + 4 * g + (e & 3) >= lt) z[e] = kNegInf;
      }
      const float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
      if (__any(top > m[t] + kMaxSlack)) {                  // (each lane its own maximum)
        const float mn = fmaxf(m[t], top);
        l[t] *= m[t] == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);
        m[t] = mn;
      }
      const float mu = m[t] == kNegInf ? 0.f : m[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) l[t] += __builtin_amdgcn_exp2f(z[e] - mu);
    }
    x = y;
    st = next;
  }
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const float mr = row_max(m[t]);
    // (a maximum of -inf beside a sum that is not 0: NaN, to be kept)
    float lr = row_sum(m[t] == kNegInf ? l[t] : l[t] * __builtin_amdgcn_exp2f(m[t] - mr));
    float mw = mr;
    if constexpr (RT == 0 && kWaves == 4) {
      if (g == 0) lds[wave * 16 + r] = mr, lds[64 + wave * 16 + r] = lr;
      __syncthreads();
      if (wave) return;
      mw = fmaxf(fmaxf(lds[r], lds[16 + r]), fmaxf(lds[32 + r], lds[48 + r]));
      lr = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float mi = lds[16 * w + r], li = lds[64 + 16 * w + r];
        lr += mi == kNegInf ? li : li * __builtin_amdgcn_exp2f(mi - mw);
      }
    }
    const int row = row0 + 16 * t + r, ti = row / a.group;
    if (g == 0 && row < it.n_rows) {
      if (it.out_row < 0) {
        sa.fin[(size_t)a.order[it.tok0 + ti] * a.heads + kvh * a.group + row - ti * a.group] = row_final(mw, lr);
      } else {
        *reinterpret_cast<float2*>(a.stat + 2 * ((size_t)it.out_row + (size_t)kvh * it.n_rows + row)) = make_float2(mw, lr);
      }
    }
  }
}

template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256) k_score_stat(ScoreArgs sa) {
  __shared__ float lds[128];
  const AttArgs& a = sa.att;
  const int n_block = a.n_kind[0] + a.n_kind[1] + a.n_kind[2];
  int item = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  if (item >= n_block) {
    const int w = (blockIdx.x - n_block * a.kv.kv_heads) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    item = n_block + w / a.kv.kv_heads;
    kvh = w % a.kv.kv_heads;
    if (item >= n_block + a.n_kind[3]) return;
  }
  const AttItem& it = a.items[item];
  // a sequence's tile whose tokens all stand before the window
  if (it.pos0 != kAllKeys && sa.back[a.order[it.tok0 + (it.n_rows - 1) / a.group]] >= sa.window) return;
  if (it.kind == 3) stat_item<E, D, FMT, 1, 0>(sa, it, kvh, lds);
  else if (it.kind == 0) stat_item<E, D, FMT, 4, 0>(sa, it, kvh, lds);
  else if (it.kind == 1) stat_item<E, D, FMT, 4, 1>(sa, it, kvh, lds);
  else if constexpr (attend_rows(sizeof(E), D) == kRowTiles[2]) stat_item<E, D, FMT, 4, 2>(sa, it, kvh, lds);
}

// The pieces of a row: 16 lanes per (token, query head).
__global__ void __launch_bounds__(256) k_score_join(ScoreArgs sa) {
  const AttArgs& a = sa.att;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  if (i >= (int64_t)a.n_joins * a.heads) return;           // (16 lanes leave together)
  const AttJoin j = a.joins[i / a.heads];
  if (sa.back[j.tok] >= sa.window) return;                 // (its pieces may not have been worked out)
  const int h = (int)(i % a.heads), kvh = h / a.group, hr = h - kvh * a.group;
  const int n = j.n[0] + j.n[1];
  float m = kNegInf, l = 0.f;
  for (int p = lane; p < n; p += 16) {
    const int k = p >= j.n[0];
    const size_t row = (size_t)(k ? j.row[1] : j.row[0]) +
                       (size_t)((k ? p - j.n[0] : p) * a.kv.kv_heads + kvh) * (k ? j.stride[1] : j.stride[0]) +
                       (k ? j.r0[1] : j.r0[0]) + hr;
    const float2 st = *reinterpret_cast<const float2*>(a.stat + 2 * row);
    const float mn = fmaxf(m, st.x);
    l = (m == kNegInf ? l : l * __builtin_amdgcn_exp2f(m - mn)) +
        (st.x == kNegInf ? st.y : st.y * __builtin_amdgcn_exp2f(st.x - mn));
    m = mn;
  }
  float top = m;
#pragma unroll
  for (int x = 1; x < 16; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
  l = m == kNegInf ? l : l * __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int x = 1; x < 16; x *= 2) l += __shfl_xor(l, x);
  if (lane == 0) sa.fin[(size_t)j.tok * a.heads + h] = row_final(top, l);
}

// 16 KT keys of one page reference and kv head to a wave, against the counted rows of their sequence that see any.
template <typename E, int D, int FMT, int KT>
__global__ void __launch_bounds__(256) k_score_add(ScoreArgs sa, int chunks) {
  const AttArgs& a = sa.att;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (the four waves of a block: runs of keys of one kv head, which read the same rows)
  const int64_t group = w / (4 * a.kv.kv_heads);
  const int kvh = (int)((w >> 2) % a.kv.kv_heads);
  const int64_t run = group * 4 + (w & 3);
  const int ref = (int)(run / chunks), first = (int)(run % chunks) * 16 * KT;
  if (ref >= sa.b.own_refs) return;
  const int count = uniform_word(sa.b.count, ref);
  if (first >= count) return;
  const SeqRec rec = sa.b.rec[uniform_word(sa.b.seq, ref)];
  if (rec.q_len == 0) return;
  const int lp = a.kv.log2_page, G = a.group;
  const int page = uniform_word(sa.b.pages, sa.b.pre_refs + ref);
  const int j0 = ((sa.b.pre_refs + ref - rec.ref0) << lp) + first;   // place of the first key in its sequence
  const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + first;
  uint32_t k[KT][D / 16];
  float ks[KT][4];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    load_words<D / 16>(a.kv.k + (vec + 16 * t) * D + lane_offset(r * D + g * (D / 4)), k[t]);
    const float4 s = *reinterpret_cast<const float4*>(a.kv.ks + vec + 16 * t + 4 * g);
    const float c = a.scale * kLog2e;
    ks[t][0] = s.x * c; ks[t][1] = s.y * c; ks[t][2] = s.z * c; ks[t][3] = s.w * c;
  }
  // rows from the first counted token on that sees the first key
  const int old = rec.len - rec.q_len;
  const int tok_a = max(max(0, rec.q_len - sa.window), j0 - old);
  float acc[KT][4] = {};
  const int rows = (rec.q_len - tok_a) * G;
  int ti = tok_a + r / G, hr = r % G;
  const int add_t = 16 / G, add_h = 16 % G;
  const E* qb = reinterpret_cast<const E*>(a.q) + (size_t)kvh * G * D + g * (D / 4);
  for (int r0 = 0; r0 < rows; r0 += 16) {
    const bool used = r0 + r < rows;
    const size_t tok = (size_t)rec.tok0 + (used ? ti : rec.q_len - 1);
    uint4 q[terms<E>()][D / 32];
    load_query<E, D>(qb + tok * a.ldq + (size_t)(used ? hr : 0) * D, used, q);
    const float2 f = used ? sa.fin[tok * a.heads + kvh * G + hr] : make_float2(0.f, 0.f);
    const int sees = used ? old + ti - j0 : -1;            // keys 0 .. sees of the run
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const f32x4 s = logits16<E, D, FMT>(k[t], q);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(s[e] * ks[t][e] - f.x) * f.y;
        acc[t][e] += 16 * t + 4 * g + e <= sees ? p : 0.f;
      }
    }
    ti += add_t;
    hr += add_h;
    if (hr >= G) hr -= G, ++ti;
  }
  // the sum over the row lanes; lane r keeps key 4 g + r % 4 of tile r / 4
  float mine = 0.f;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = acc[t][e];
#pragma unroll
      for (int x = 1; x < 16; x *= 2) v += __shfl_xor(v, x);
      if (r == 4 * t + e) mine = v;
    }
  const int at = 16 * (r >> 2) + 4 * g + (r & 3);
  if (r < 4 * KT && first + at < count) {
    const int j = j0 + at, fresh = j - old;                 // (>= 0: the step's own token)
    const float had = fresh >= 0 ? 0.f : a.kv.weight[vec + at];
    a.kv.weight[vec + at] = had + mine;
    if (fresh >= 0) a.kv.place[vec + at] = sa.pos ? sa.pos[rec.tok0 + fresh] : j;
  }
}

// Marks out of the cache or into it: a block takes one page reference.
template <bool kWrite>
__global__ void __launch_bounds__(256) k_marks(MarksArgs a) {
  const int ref = blockIdx.x, hk = a.kv.kv_heads;
  const int count = a.b.count[ref];
  const int64_t row = a.b.row[ref];
  const size_t page = a.b.pages[a.b.pre_refs + ref];
  for (int i = threadIdx.x; i < count * hk; i += 256) {
    const int at = i / hk, h = i - at * hk;
    const size_t in = ((page * hk + h) << a.kv.log2_page) + at, out = (size_t)row * hk + i;
    if (kWrite) {
      a.kv.weight[in] = a.weight[out];
      a.kv.place[in] = a.place[out];
    } else {
      a.weight[out] = a.kv.weight[in];
      a.place[out] = a.kv.place[in];
    }
  }
}

// ---- eviction ------------------------------------------------------------------------------
// One (sequence, kv head) to a block.  Of n > keep tokens those stay that come first by: position among the
// `recent` newest; weight, larger ones first, NaN above all; place, lower ones first.  The number that a token
// orders by is 32 bits wide; a radix select (11, 11 and 10 bits, histograms in LDS) finds the keep-th
// largest, a bit for each token says which stay, and the kept ones behind place `keep` go to
// the places of the dropped ones before it, in order.  No two moves touch one place.
constexpr uint32_t kProtected = 0xffffffffu, kNanKey = 0xfffffffeu;
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return kNanKey;
  const uint32_t u = __float_as_uint(w + 0.f);             // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr int kBins = 2048, kMoves = 2048;                 // moves listed at a time

struct alignas(16) EvictLds {                                          // dynamic LDS: keys (kept where they fit), bits, and these
  uint32_t hist[kBins];
  int32_t hole[kMoves], mover[kMoves];
  int32_t wave[16], wave2[16];
  int32_t newest;
  uint32_t prefix;
  int32_t need;
};

template <int NT>   // threads
__global__ void __launch_bounds__(NT) k_evict(EvictArgs a, int cached) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  EvictLds& sh = *reinterpret_cast<EvictLds*>(dyn);
  uint32_t* bits = reinterpret_cast<uint32_t*>(dyn + sizeof(EvictLds));
  uint32_t* keys = bits + (a.max_len + 63) / 64 * 2;       // (cached: room for max_len keys)
  const int seq = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  const SeqRec rec = a.b.rec[seq];
  const int n = rec.len, keep = a.keep, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  constexpr int kWaves = NT / 64;
  if (n <= keep) return;
  const int lp = a.kv.log2_page, hk = a.kv.kv_heads;
  const int32_t* pages = a.b.pages + rec.ref0;
  auto vec_of = [&](int j) { return (((size_t)pages[j >> lp] * hk + kvh) << lp) + (j & ((1 << lp) - 1)); };
  // the newest position
  if (tid == 0) sh.newest = INT32_MIN;
  __syncthreads();
  if (a.recent > 0) {
    int top = INT32_MIN;
    for (int j = tid; j < n; j += NT) top = max(top, a.kv.place[vec_of(j)]);
    for (int i = 1; i < 64; i *= 2) top = max(top, __shfl_xor(top, i));
    if (lane == 0) atomicMax(&sh.newest, top);
    __syncthreads();
  }
  const int64_t since = a.recent > 0 ? (int64_t)sh.newest - a.recent : INT64_MAX;
  auto key_at = [&](int j) {
    const size_t v = vec_of(j);
    const uint32_t k = weight_order(a.kv.weight[v]);
    return a.recent > 0 && (int64_t)a.kv.place[v] > since ? kProtected : k;
  };
  if (cached)
    for (int j = tid; j < n; j += NT) keys[j] = key_at(j);
  auto key_of = [&](int j) { return cached ? keys[j] : key_at(j); };
  // the keep-th largest key: `prefix`, of which `need` stay
  uint32_t prefix = 0;
  int need = keep;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += NT) sh.hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += NT) {
      const uint32_t k = key_of(j);
      if (pass == 0 || (k >> (shift + width)) == (prefix >> (shift + width)))
        atomicAdd(&sh.hist[(k >> shift) & ((1u << width) - 1u)], 1u);
    }
    __syncthreads();
    // wave 0: each lane the sum of 32 bins, the largest in lane 0; then the bins of the lane that `need` falls to
    if (wv == 0) {
      uint32_t sum = 0;
      for (int i = 0; i < 32; ++i) sum += sh.hist[kBins - 1 - (lane * 32 + i)];
      uint32_t upto = sum;
      for (int i = 1; i < 64; i *= 2) {
        const uint32_t o = __shfl_up(upto, i);
        upto += lane >= i ? o : 0u;
      }
      const uint64_t who = __ballot(upto >= (uint32_t)need);
      if (lane == __builtin_ctzll(who)) {                  // (n > keep >= need: one has it; need = 0: lane 0)
        uint32_t before = upto - sum;
        int b = kBins - 1 - lane * 32;
        while (before + sh.hist[b] < (uint32_t)need) before += sh.hist[b--];
        sh.prefix = prefix | ((uint32_t)b << shift);
        sh.need = need - (int)before;
      }
    }
    __syncthreads();
    prefix = sh.prefix;
    need = sh.need;
  }
  // Every wave a run of whole words of bits: how many equal the keep-th, then which stay.
  const int words = (n + 63) / 64, per = (words + kWaves - 1) / kWaves;
  const int w0 = min(wv * per, words), w1 = min(w0 + per, words);
  auto before_wave = [&](int32_t* s, int mine) {
    if (lane == 0) s[wv] = mine;
    __syncthreads();
    int sum = 0;
    for (int i = 0; i < wv; ++i) sum += s[i];
    return sum;
  };
  int equal = 0;
  for (int w = w0; w < w1; ++w) {
    const int j = w * 64 + lane;
    equal += __popcll(__ballot(j < n && key_of(j) == prefix));
  }
  equal = before_wave(sh.wave, equal);
  int holes = 0, movers = 0;
  const uint64_t below = (1ull << lane) - 1;
  for (int w = w0; w < w1; ++w) {
    const int j = w * 64 + lane;
    const uint32_t k = j < n ? key_of(j) : 0u;
    const uint64_t same = __ballot(j < n && k == prefix);
    const bool stays = j < n && (k > prefix || (k == prefix && equal + __popcll(same & below) < need));
    equal += __popcll(same);
    const uint64_t kept = __ballot(stays);
    if (lane == 0) reinterpret_cast<uint64_t*>(bits)[w] = kept;
    holes += __popcll(__ballot(j < keep && !stays));
    movers += __popcll(__ballot(j >= keep && stays));
  }
  __syncthreads();
  const int hole0 = before_wave(sh.wave, holes), mover0 = before_wave(sh.wave2, movers);
  int total = 0;
  for (int i = 0; i < kWaves; ++i) total += sh.wave[i];    // (as many movers)
  for (int first = 0; first < total; first += kMoves) {
    __syncthreads();
    int h = hole0 - first, m = mover0 - first;
    for (int w = w0; w < w1; ++w) {
      const int j = w * 64 + lane;
      const uint64_t kept = reinterpret_cast<const uint64_t*>(bits)[w];
      const bool stays = (kept >> lane) & 1;
      const uint64_t hs = __ballot(j < keep && !stays), ms = __ballot(j >= keep && j < n && stays);
      const int hi = h + __popcll(hs & below), mi = m + __popcll(ms & below);
      if (((hs >> lane) & 1) && hi >= 0 && hi < kMoves) sh.hole[hi] = j;
      if (((ms >> lane) & 1) && mi >= 0 && mi < kMoves) sh.mover[mi] = j;
      h += __popcll(hs);
      m += __popcll(ms);
    }
    __syncthreads();
    const int todo = min(kMoves, total - first), dv = a.kv.dim / 16;
    for (int i = tid; i < todo * 2 * dv; i += NT) {
      const int mv = i / (2 * dv), part = i - mv * 2 * dv;
      const size_t from = vec_of(sh.mover[mv]), to = vec_of(sh.hole[mv]);
      uint8_t* p = part < dv ? a.kv.k : a.kv.v;
      const int o = (part < dv ? part : part - dv) * 16;
      *reinterpret_cast<uint4*>(p + to * a.kv.dim + o) = *reinterpret_cast<const uint4*>(p + from * a.kv.dim + o);
    }
    for (int i = tid; i < todo; i += NT) {
      const size_t from = vec_of(sh.mover[i]), to = vec_of(sh.hole[i]);
      a.kv.ks[to] = a.kv.ks[from];
      a.kv.vs[to] = a.kv.vs[from];
      a.kv.weight[to] = a.kv.weight[from];
      a.kv.place[to] = a.kv.place[from];
    }
  }
}

template <typename E, int D, int FMT>
void score_typed(const ScoreArgs& sa, hipStream_t s) {
  const AttArgs& a = sa.att;
  const int blocks = (a.n_kind[0] + a.n_kind[1] + a.n_kind[2]) * a.kv.kv_heads + cdiv(a.n_kind[3] * a.kv.kv_heads, 4);
  hipLaunchKernelGGL((k_score_stat<E, D, FMT>), dim3(blocks), dim3(256), 0, s, sa);
  if (a.n_joins)
    hipLaunchKernelGGL(k_score_join, dim3((unsigned)(((int64_t)a.n_joins * a.heads + 15) / 16)), dim3(256), 0, s, sa);
  auto add = [&](auto kt) {
    constexpr int KT = decltype(kt)::value;
    if (sa.b.own_refs == 0) return;
    const int page = 1 << a.kv.log2_page;
    hipLaunchKernelGGL((k_score_add<E, D, FMT, KT>), dim3((unsigned)score_blocks(sa.b.own_refs, page, a.kv.kv_heads)),
                       dim3(256), 0, s, sa, page / score_run(page));
  };
  if (score_run(1 << a.kv.log2_page) == 16) add(std::integral_constant<int, 1>());
  else if (score_run(1 << a.kv.log2_page) == 32) add(std::integral_constant<int, 2>());
  else add(std::integral_constant<int, 4>());
}
template <typename E, int D>
void score_format(const ScoreArgs& a, hipStream_t s) {
  if (a.att.kv.format == kKvInt8) score_typed<E, D, kKvInt8>(a, s);
  else score_typed<E, D, kKvE4m3>(a, s);
}
template <typename E>
void score_dim(const ScoreArgs& a, hipStream_t s) {
  if (a.att.kv.dim == 64) score_format<E, 64>(a, s);
  else if (a.att.kv.dim == 128) score_format<E, 128>(a, s);
  else score_format<E, 256>(a, s);
}

}  // namespace

hipError_t launch_score(const ScoreArgs& a, int bf16, hipStream_t s) {
  if (bf16) score_dim<uint16_t>(a, s);
  else score_dim<float>(a, s);
  return hipGetLastError();
}

hipError_t launch_marks(const MarksArgs& a, bool write, hipStream_t s) {
  if (write) hipLaunchKernelGGL(k_marks<true>, dim3(a.b.own_refs), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_marks<false>, dim3(a.b.own_refs), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  const int bits = (a.max_len + 63) / 64 * 8;
  const int cached = a.max_len <= 16384;
  const int lds = (int)sizeof(EvictLds) + bits + (cached ? a.max_len * 4 : 0);
  const dim3 grid((unsigned)((int64_t)a.b.n_seqs * a.kv.kv_heads));
  if (a.max_len <= 4096) hipLaunchKernelGGL(k_evict<256>, grid, dim3(256), lds, s, a, cached);
  else hipLaunchKernelGGL(k_evict<1024>, grid, dim3(1024), lds, s, a, cached);
  return hipGetLastError();
}

}  // namespace salt
