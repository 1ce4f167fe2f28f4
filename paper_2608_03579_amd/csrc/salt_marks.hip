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
// the second goes by keys and adds up exp2(logit - maximum) / sum over the rows (k_score_few, k_score_many): every
// mark has one owner and is written once, so no atomics, and the sum's order is fixed.
// Codes are exact in bf16; q enters as it is in bf16 contexts, in three bf16 terms (24 bits) in fp32 ones.
// The attention itself has the maxima and sums, but keeps them in its work items; taking them from there would tie a
// layer's score to its attention.  Measured with 32 heads in 8 groups, a kernel by itself under the profiler, on inputs
// repeated: 64 sequences of up to 4096 keys, one token each, 11.8 + 10.8 us (31 MB of keys read twice, the second time
// from the Infinity Cache); two prompts of 4096 tokens, 215 + 230 us for 2 x 137 GFLOP, 64 + 16 where their last 64 tokens
// count; in fp32 423 + 567, of heads of 256 1041 + 1110.  The calls on fresh inputs, marks in and out among them: 28 and
// 392 us.
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

// A vector's values that lane group g brings to the products are a run of dim / 4 from dim / 4 g on.
template <typename E, int D>
__device__ __forceinline__ void load_query(const E* q, int g, bool used, uint4 (&o)[terms<E>()][D / 32]) {
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    const E* at = q + g * (D / 4) + 8 * ks;
    if constexpr (sizeof(E) == 2) {
      o[0][ks] = used ? *reinterpret_cast<const uint4*>(at) : make_uint4(0u, 0u, 0u, 0u);
    } else {
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (used) load8(at, f);
      uint4 t[terms<E>()];
      split_terms<terms<E>()>(f, t);
#pragma unroll
      for (int n = 0; n < terms<E>(); ++n) o[n][ks] = t[n];
    }
  }
}

// What the wave's lanes wrote to LDS before is there for all of them after.  (LDS keeps a wave's order: the compiler has to.)
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Rows of kBytes that a wave stages in LDS of its own.  An operand load straight from memory gives neighbouring lanes
// neighbouring rows: 64 cache lines to an instruction, which the address unit takes a cycle each for (rows of q read so:
// k_score_many 330 us on the prompts above, 107 with its loads left out).  From here the wave reads memory in order,
// 1 KB to an instruction, and LDS as the operand needs it.  Chunks of 16 bytes change places within their row so
// that 16 rows' chunks fall into different banks.
template <int kBytes>
struct Staged {
  static constexpr int kChunks = kBytes / 16;              // of a row
  static __device__ __forceinline__ int at(int row, int chunk) {
    constexpr int kWindow = kChunks < 16 ? 16 / kChunks : 1;   // rows that 256 bytes hold
    return row * kBytes + 16 * (chunk ^ ((row / kWindow) & (kChunks - 1) & 15));
  }
  // The lane's row and chunk in load j of 64 chunks.
  static __device__ __forceinline__ int row(int j, int lane) { return (j * 64 + lane) / kChunks; }
  static __device__ __forceinline__ int chunk(int j, int lane) { return (j * 64 + lane) % kChunks; }
};

// 16 keys' codes as the products' operand.
template <int D, int FMT>
__device__ __forceinline__ void keys_bf16(const uint32_t (&k)[D / 16], uint4 (&o)[D / 32]) {
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) {
    const uint2 lo = codes_bf16<FMT>(k[2 * ks]), hi = codes_bf16<FMT>(k[2 * ks + 1]);
    o[ks] = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
}
// Products of 16 keys (the lane: keys 4 g + i) and 16 rows (row l & 15).
template <typename E, int D>
__device__ __forceinline__ f32x4 products16(const uint4 (&k)[D / 32], const uint4 (&q)[terms<E>()][D / 32]) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
    for (int n = 0; n < terms<E>(); ++n) s = mma_bf16(k[ks], q[n][ks], s);
  return s;
}

// 32 keys of an item as they come from memory, 16 and 16 in a row, and through LDS as operands: keys (l & 15) and
// 16 + (l & 15), a run of dim / 4 codes each.
template <int D>
struct Keys32 {
  u32x4 c[2][D / 64];
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
  const int lp = a.kv.log2_page, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int j = min(x.j0 + 16 * t, last & ~15);         // a run of 16 keys lies in one page
    const int page = uniform_word(a.pages, ref + (j >> lp));
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    const uint8_t* k = a.kv.k + vec * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) x.c[t][i] = *reinterpret_cast<const u32x4*>(k + lane_offset(i * 1024 + lane * 16));
    const float4 s = *reinterpret_cast<const float4*>(a.kv.ks + vec + (uint32_t)(4 * g));
    x.ks[4 * t] = s.x; x.ks[4 * t + 1] = s.y; x.ks[4 * t + 2] = s.z; x.ks[4 * t + 3] = s.w;
  }
}
// 16 keys into the wave's LDS, and out of it.
template <int D>
__device__ __forceinline__ void stage_keys(uint8_t* lds, int lane, const u32x4 (&c)[D / 64]) {
  using S = Staged<D>;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) *reinterpret_cast<u32x4*>(lds + S::at(S::row(i, lane), S::chunk(i, lane))) = c[i];
}
template <int D>
__device__ __forceinline__ void read_keys(const uint8_t* lds, int lane, uint32_t (&w)[D / 16]) {
  const int r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + Staged<D>::at(r, g * (D / 64) + i));
    w[4 * i] = v[0]; w[4 * i + 1] = v[1]; w[4 * i + 2] = v[2]; w[4 * i + 3] = v[3];
  }
}

// What a row's exponentials are multiplied by: 1 / sum.  A sum of 0: no key has a logit above -inf, and the
// weights are NaN, as the formula's.
__device__ __forceinline__ float2 row_final(float m, float l) {
  return make_float2(m == kNegInf ? 0.f : m, l == 0.f ? __builtin_nanf("") : 1.0f / l);
}

// One item: RT row tiles of 16 to a wave, WR waves side by side over the rows and WK over the keys, 32 keys in turn.
// (WK = WR = 1: one wave alone.)  Each lane has a running maximum and sum of its own keys, joined over lanes and
// waves in the end.  A logit is an fma against the maximum so far, which follows the largest one only when that
// is kMaxSlack above it.  Few rows are bound by latency.  Many keep the vector unit busy for 58 % of the time (27
// instructions to 16 keys x 16 rows, four of them exponentials at a quarter of the rate) and the matrix unit for 29 %; the
// rest are waits of two waves to a SIMD.  Four row tiles to a wave where registers allow: codes are converted once for
// all (two tiles: 237 to 269 us for 215), and one test for all of them whether a maximum has to follow (a test for each: 240 us).
template <typename E, int D, int FMT, int RT, int WR, int WK>
__device__ __forceinline__ void stat_item(const ScoreArgs& sa, const AttItem& it, int kvh, uint8_t* stage, float* lds) {
  const AttArgs& a = sa.att;
  constexpr int NT = terms<E>();
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = WR * WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int n_pre = 2 * ((it.pre_len + kKeyUnit - 1) / kKeyUnit);
  const int row0 = wr * 16 * RT;
  const bool on = row0 < it.n_rows;                        // (a tile may be short of rows)
  int st = 2 * it.unit0 + wk;
  const int st1 = on ? 2 * it.unit1 : 0;
  Keys32<D> x;
  if (st < st1) load_keys32<D>(a, it, n_pre, st, kvh, lane, x);
  uint4 q[RT][NT][D / 32];
  float m[RT], l[RT], bar[RT];                             // bar: how far above m a logit may be; -inf: m is not yet set
  int lim[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = row0 + 16 * t + r, ti = row / a.group;
    const bool used = row < it.n_rows;
    const int tok = used ? a.order[it.tok0 + ti] : 0;
    load_query<E, D>(reinterpret_cast<const E*>(a.q) + (size_t)tok * a.ldq +
                               (size_t)(kvh * a.group + row - ti * a.group) * D, g, used, q[t]);
    m[t] = 0.f;
    l[t] = 0.f;
    bar[t] = kNegInf;
    lim[t] = it.pos0 + ti + 1;
  }
  const int min_lim = it.pos0 + row0 / a.group + 1;
  const float c = a.scale * kLog2e;
  auto use = [&](const Keys32<D>& x) {
    const bool edge = x.j0 + 32 > (x.own ? min_lim : x.end);
    uint4 k[2][D / 32];
    float ks[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t w[D / 16];
      read_keys<D>(stage + u * 16 * D, lane, w);
      keys_bf16<D, FMT>(w, k[u]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ks[e] = x.ks[e] * c;
    float z[RT][8], top[RT];
    bool above = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x4 s = products16<E, D>(k[u], q[t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[t][4 * u + e] = fmaf(s[e], ks[4 * u + e], -m[t]);
      }
    }
    if (edge) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int lt = x.own ? min(lim[t], x.end) : x.end;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (x.j0 + 16 * (e >> 2) + 4 * g + (e & 3) >= lt) z[t][e] = kNegInf;
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      top[t] = max3_of(max3_of(max3_of(z[t][0], z[t][1], z[t][2]), z[t][3], z[t][4]), max3_of(z[t][5], z[t][6], z[t][7]), z[t][7]);
      above |= top[t] > bar[t];
    }
    if (__any(above)) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float up = top[t] > bar[t] ? top[t] : 0.f;
        if (bar[t] > kNegInf) l[t] *= __builtin_amdgcn_exp2f(-up);
        if (top[t] > bar[t]) bar[t] = kMaxSlack;
        m[t] += up;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[t][e] -= up;
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) l[t] += __builtin_amdgcn_exp2f(z[t][e]);
  };
  auto put = [&](const Keys32<D>& x) {
    wave_order();                                          // (the keys before have been read)
#pragma unroll
    for (int u = 0; u < 2; ++u) stage_keys<D>(stage + u * 16 * D, lane, x.c[u]);
    wave_order();
  };
  Keys32<D> y;
  for (; st < st1; st += 2 * WK) {
    put(x);
    if (st + WK < st1) load_keys32<D>(a, it, n_pre, st + WK, kvh, lane, y);
    use(x);
    if (st + WK >= st1) break;
    put(y);
    if (st + 2 * WK < st1) load_keys32<D>(a, it, n_pre, st + 2 * WK, kvh, lane, x);
    use(y);
  }
  constexpr int kRows = 16 * RT * WR;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (bar[t] == kNegInf) m[t] = kNegInf;
    const float mr = row_max(m[t]);
    // (a maximum of -inf beside a sum that is not 0: NaN, to be kept)
    l[t] = row_sum(m[t] == kNegInf ? l[t] : l[t] * __builtin_amdgcn_exp2f(m[t] - mr));
    m[t] = mr;
    if constexpr (WK > 1)
      if (g == 0) {
        const int at = wk * kRows + row0 + 16 * t + r;
        lds[at] = m[t];
        lds[WK * kRows + at] = l[t];
      }
  }
  if constexpr (WK > 1) {
    __syncthreads();
    if (wk) return;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = row0 + 16 * t + r, ti = row / a.group;
    float mw = m[t], lr = l[t];
    if constexpr (WK > 1) {
#pragma unroll
      for (int w = 1; w < WK; ++w) mw = fmaxf(mw, lds[w * kRows + row]);
      lr = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const float mi = lds[w * kRows + row], li = lds[(WK + w) * kRows + row];
        lr += mi == kNegInf ? li : li * __builtin_amdgcn_exp2f(mi - mw);
      }
    }
    if (g == 0 && row < it.n_rows) {
      if (it.out_row < 0) {
        sa.fin[(size_t)a.order[it.tok0 + ti] * a.heads + kvh * a.group + row - ti * a.group] = row_final(mw, lr);
      } else {
        *reinterpret_cast<float2*>(a.stat + 2 * ((size_t)it.out_row + (size_t)kvh * it.n_rows + row)) = make_float2(mw, lr);
      }
    }
  }
}

// Row tiles of a wave: what 96 registers of q hold, four at most.
template <typename E, int D>
constexpr int row_tiles() {
  constexpr int n = 96 * 8 / (terms<E>() * D);
  return n >= 4 ? 4 : n >= 2 ? 2 : 1;
}

template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256, sizeof(E) * D <= 256 ? 2 : 1) k_score_stat(ScoreArgs sa) {
  __shared__ float lds[512];
  __shared__ __attribute__((aligned(16))) uint8_t staged[4][32 * D];
  const AttArgs& a = sa.att;
  uint8_t* stage = staged[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
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
  constexpr int RT = row_tiles<E, D>();
  if (it.kind == 3) stat_item<E, D, FMT, 1, 1, 1>(sa, it, kvh, stage, lds);
  else if (it.kind == 0) stat_item<E, D, FMT, 1, 1, 4>(sa, it, kvh, stage, lds);
  else if (it.kind == 1) stat_item<E, D, FMT, RT, 4 / RT, RT>(sa, it, kvh, stage, lds);
  else if constexpr (attend_rows(sizeof(E), D) == kRowTiles[2]) stat_item<E, D, FMT, RT, 8 / RT, RT / 2>(sa, it, kvh, stage, lds);
}

// Entry i of p, for a wave-uniform i: by way of the scalar unit.  (p is not written by this launch.)
template <typename S>
__device__ __forceinline__ S uniform_entry(const S* p, int i) {
  constexpr int kWords = sizeof(S) / 4;
  struct Words {
    int32_t w[kWords];
  } v;
  const auto* w = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(p + __builtin_amdgcn_readfirstlane(i));
#pragma unroll
  for (int k = 0; k < kWords; ++k) v.w[k] = w[k];
  return __builtin_bit_cast(S, v);
}
// A joined row's partial result of piece p.
__device__ __forceinline__ float2 piece_of(const AttArgs& a, const AttJoin& j, int p, int kvh, int hr) {
  const int k = p >= j.n[0];
  const size_t row = (size_t)(k ? j.row[1] : j.row[0]) +
                     (size_t)((k ? p - j.n[0] : p) * a.kv.kv_heads + kvh) * (k ? j.stride[1] : j.stride[0]) +
                     (k ? j.r0[1] : j.r0[0]) + hr;
  return *reinterpret_cast<const float2*>(a.stat + 2 * row);
}
__device__ __forceinline__ void join_piece(float& m, float& l, float2 st) {
  const float mn = fmaxf(m, st.x);
  l = (m == kNegInf ? l : l * __builtin_amdgcn_exp2f(m - mn)) +
      (st.x == kNegInf ? st.y : st.y * __builtin_amdgcn_exp2f(st.x - mn));
  m = mn;
}

// The pieces of a row, for sequences of many rows: 16 lanes per (token, query head).
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
  for (int p = lane; p < n; p += 16) join_piece(m, l, piece_of(a, j, p, kvh, hr));
  float top = m;
#pragma unroll
  for (int x = 1; x < 16; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
  l = m == kNegInf ? l : l * __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int x = 1; x < 16; x *= 2) l += __shfl_xor(l, x);
  if (lane == 0) sa.fin[(size_t)j.tok * a.heads + h] = row_final(top, l);
}

// A unit of 64 own keys of one sequence, as one wave has it: bf16 codes and scales times the logits' factor.
template <int D>
struct Unit {
  int j0;                  // place of the first key
  uint4 k[4][D / 32];
  float ks[4][4];
};
template <int D>
struct UnitCodes {
  u32x4 c[4][D / 64];
  float4 s[4];
};
template <int D>
__device__ __forceinline__ void load_unit(const ScoreArgs& sa, int j0, const SeqRec& rec, int kvh, UnitCodes<D>& x) {
  const AttArgs& a = sa.att;
  const int lane = threadIdx.x & 63, g = lane >> 4, lp = a.kv.log2_page;
  // the unit's pages, looked up at once: one, or four references in a row (those past the sequence's last are not used)
  struct Refs {
    int32_t page[4];
  } refs{};
  const int first = rec.ref0 + (j0 >> lp);
  if (lp >= 6) refs.page[0] = uniform_word(a.pages, first);
  else refs = uniform_entry(reinterpret_cast<const Refs*>(a.pages + first), 0);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int j = min(j0 + 16 * t, (rec.len - 1) & ~15);   // a run of 16 keys lies in one page
    const int ref = (j >> lp) - (j0 >> lp);
    const int page = ref == 0 ? refs.page[0] : ref == 1 ? refs.page[1] : ref == 2 ? refs.page[2] : refs.page[3];
    const size_t vec = (((size_t)page * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
    const uint8_t* k = a.kv.k + vec * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) x.c[t][i] = *reinterpret_cast<const u32x4*>(k + lane_offset(i * 1024 + lane * 16));
    x.s[t] = *reinterpret_cast<const float4*>(a.kv.ks + vec + 4 * g);
  }
}
template <int D, int FMT>
__device__ __forceinline__ void convert_unit(const UnitCodes<D>& u, float c, int j0, uint8_t* stage, Unit<D>& x) {
  const int lane = threadIdx.x & 63;
  x.j0 = j0;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    x.ks[t][0] = u.s[t].x * c; x.ks[t][1] = u.s[t].y * c; x.ks[t][2] = u.s[t].z * c; x.ks[t][3] = u.s[t].w * c;
    uint32_t w[D / 16];
    stage_keys<D>(stage + (t & 1) * 16 * D, lane, u.c[t]);   // (LDS keeps a wave's order)
    wave_order();
    read_keys<D>(stage + (t & 1) * 16 * D, lane, w);
    wave_order();
    keys_bf16<D, FMT>(w, x.k[t]);
  }
}
// The first counted token that sees the unit's first key.
__device__ __forceinline__ int first_token(const ScoreArgs& sa, const SeqRec& rec, int j0) {
  return max(max(0, rec.q_len - sa.window), j0 - (rec.len - rec.q_len));
}
// The sum over the 16 lanes of a row of lanes, in all of them.
template <int N>
__device__ __forceinline__ float add_turned(float v) {       // row_ror:N
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, true));
}
// The weights' sums over the 16 row lanes: lane r gets key 4 g + r % 4 of tile r / 4.
__device__ __forceinline__ float sum_rows(const float (&acc)[4][4]) {
  const int r = threadIdx.x & 15;
  float mine = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float v = add_turned<1>(add_turned<2>(add_turned<4>(add_turned<8>(acc[i >> 2][i & 3]))));
    mine = r == i ? v : mine;
  }
  return mine;
}
// Key `at` of the unit has gathered `w` in this step.
__device__ __forceinline__ void add_mark(const ScoreArgs& sa, const SeqRec& rec, int j, int kvh, float w) {
  const AttArgs& a = sa.att;
  if (j >= rec.len) return;
  const int lp = a.kv.log2_page;
  const size_t vec = (((size_t)a.pages[rec.ref0 + (j >> lp)] * a.kv.kv_heads + kvh) << lp) + (j & ((1 << lp) - 1));
  const int fresh = j - (rec.len - rec.q_len);             // (>= 0: the step's own token)
  const float had = fresh >= 0 ? 0.f : a.kv.weight[vec];
  a.kv.weight[vec] = had + w;
  if (fresh >= 0) a.kv.place[vec] = sa.pos ? sa.pos[rec.tok0 + fresh] : j;
}

// 16 rows against the unit, each key for the rows that see it (kEdge), or for all.
template <typename E, int D, bool kEdge>
__device__ __forceinline__ void add_rows(const Unit<D>& x, const uint4 (&q)[terms<E>()][D / 32], float2 f, int sees,
                                         float (&acc)[4][4]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const f32x4 s = products16<E, D>(x.k[t], q);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[e], x.ks[t][e], -f.x));
      if (kEdge) acc[t][e] += 16 * t + 4 * g + e <= sees ? p * f.y : 0.f;
      else acc[t][e] = fmaf(p, f.y, acc[t][e]);
    }
  }
}

// Sequences of few counted rows: a wave to a unit and kv head.  The rows' pieces are joined here, by every wave again: a
// launch less (4.3 us).  Bound by its chain of dependent reads (unit, sequence, pages, keys, pieces) and by some 156
// registers, three waves to a SIMD; held to 128 it spills (14.3 us for 10.8).
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256, sizeof(E) * D <= 256 ? 2 : 1) k_score_few(ScoreArgs sa) {
  const AttArgs& a = sa.att;
  __shared__ __attribute__((aligned(16))) uint8_t staged[4][32 * D];
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, G = a.group;
  // (the four waves of a block: units of one kv head)
  const int kvh = blockIdx.x % a.kv.kv_heads;
  const int unit = (blockIdx.x / a.kv.kv_heads) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= sa.b.n_units) return;
  const SeqRec rec = uniform_entry(sa.b.rec, uniform_word(sa.b.unit, unit));
  if (rec.q_len == 0 || (int64_t)min(rec.q_len, sa.window) * G > kFewRows) return;
  const int j0 = (unit - rec.unit0) * kKeyUnit, old = rec.len - rec.q_len;
  UnitCodes<D> codes;
  load_unit<D>(sa, j0, rec, kvh, codes);
  int tok_a = __builtin_amdgcn_readfirstlane(first_token(sa, rec, j0));
  asm volatile("" : "+s"(tok_a));                          // (the keys are on their way before the rest is looked up)
  const int rows = (rec.q_len - tok_a) * G;
  // Of a single token the join comes by the scalar unit, which does not wait for the keys.
  const bool one = rec.q_len - tok_a == 1;
  int join1 = -1;
  AttJoin j1{};
  if (one) {
    join1 = uniform_word(sa.joined, rec.tok0 + tok_a);
    if (join1 >= 0) j1 = uniform_entry(a.joins, join1);
  }
  Unit<D> x;
  convert_unit<D, FMT>(codes, a.scale * kLog2e, j0, staged[threadIdx.x >> 6], x);
  float acc[4][4] = {};
  const E* qb = reinterpret_cast<const E*>(a.q) + (size_t)kvh * G * D;
  for (int r0 = 0; r0 < rows; r0 += 16) {
    const bool used = r0 + r < rows;
    const int row = used ? r0 + r : 0, ti = tok_a + row / G, hr = row % G;
    const size_t tok = (size_t)rec.tok0 + ti;
    uint4 q[terms<E>()][D / 32];
    load_query<E, D>(qb + tok * a.ldq + (size_t)hr * D, g, used, q);
    const int join = one ? join1 : sa.joined[tok];
    const AttJoin j = one ? j1 : join >= 0 ? a.joins[join] : AttJoin{};
    const int n = join >= 0 ? j.n[0] + j.n[1] : 0;
    float m = kNegInf, l = 0.f;
    for (int p = g; p < n; p += 4) join_piece(m, l, piece_of(a, j, p, kvh, hr));   // (a row's four lanes share them)
    const float top = row_max(m);
    l = row_sum(m == kNegInf ? l : l * __builtin_amdgcn_exp2f(m - top));
    const float2 f = join >= 0 ? row_final(top, l) : sa.fin[tok * a.heads + kvh * G + hr];
    add_rows<E, D, true>(x, q, f, used ? old + ti - x.j0 : -1, acc);
  }
  const float w = sum_rows(acc);
  add_mark(sa, rec, x.j0 + 16 * (r >> 2) + 4 * g + (r & 3), kvh, w);
}

// Sequences of many counted rows: a block to a unit and kv head, whose waves take 16 rows in turn, the next ones on
// their way; their sums meet in LDS.  Bound by waits for rows and LDS that two waves to a SIMD do not hide: the vector unit
// (75 instructions to 64 keys x 16 rows) is busy for 39 % of the time, the matrix unit for 28 %.  A wave to a unit, rows
// not shared out: 911 us for 230.
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256, sizeof(E) * D <= 256 ? 2 : 1) k_score_many(ScoreArgs sa) {
  const AttArgs& a = sa.att;
  using S = Staged<D * sizeof(E)>;
  constexpr int kStage = 16 * D * (int)sizeof(E);          // 16 rows, or 32 keys
  __shared__ __attribute__((aligned(16))) uint8_t staged[4][kStage];
  __shared__ float sums[4][kKeyUnit];
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, G = a.group;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t* stage = staged[wave];
  const int kvh = blockIdx.x % a.kv.kv_heads, unit = blockIdx.x / a.kv.kv_heads;
  const SeqRec rec = uniform_entry(sa.b.rec, uniform_word(sa.b.unit, unit));
  if (rec.q_len == 0 || (int64_t)min(rec.q_len, sa.window) * G <= kFewRows) return;
  const int j0 = (unit - rec.unit0) * kKeyUnit;
  UnitCodes<D> codes;
  load_unit<D>(sa, j0, rec, kvh, codes);
  Unit<D> x;
  convert_unit<D, FMT>(codes, a.scale * kLog2e, j0, stage, x);
  const int old = rec.len - rec.q_len, tok_a = first_token(sa, rec, j0);
  float acc[4][4] = {};
  // A tile is as many whole tokens as have 16 rows (of groups above 16: a token's rows 16 at a time), so that a lane's
  // rows lie at fixed offsets from the tile's first.  The last ones first: blocks of all units that run at a time then
  // read the same rows, which stay in the L2 cache.
  const int toks = rec.q_len - tok_a;
  const int per = G <= 16 ? 16 / G : 1, parts = G <= 16 ? 1 : (G + 15) / 16;
  const int tiles = (toks + per - 1) / per * parts, full = toks / per * parts;
  // tokens that do not see the unit's last key, and the first tile without any of them
  const int some = min(max(j0 + kKeyUnit - 1 - old - tok_a, 0), toks);
  const int plain = min(full, (some + per - 1) / per * parts);
  const char* qb = reinterpret_cast<const char*>(reinterpret_cast<const E*>(a.q) + ((size_t)rec.tok0 + tok_a) * a.ldq + (size_t)kvh * G * D);
  const float2* fb = sa.fin + ((size_t)rec.tok0 + tok_a) * a.heads + kvh * G;
  const uint32_t row_bytes = D * sizeof(E), tok_bytes = (uint32_t)a.ldq * (uint32_t)sizeof(E);   // (ldq <= kScoreRow)
  // row k of a tile of `n` rows whose heads begin at h0: its token and head
  auto place = [&](int k, int n, int h0, int& ti, int& hr) {
    k = min(k, n - 1);
    ti = G <= 16 ? k / G : 0;
    hr = G <= 16 ? k - ti * G : h0 + k;
  };
  uint32_t off[S::kChunks / 4], f_off;
  int my_ti = 0;
  auto offsets = [&](int n, int h0) {
    int ti, hr;
#pragma unroll
    for (int k = 0; k < S::kChunks / 4; ++k) {
      place(S::row(k, lane), n, h0, ti, hr);
      off[k] = ti * tok_bytes + hr * row_bytes + 16 * S::chunk(k, lane);
    }
    place(r, n, h0, ti, hr);
    f_off = ti * a.heads + hr;
    my_ti = ti;
  };
  u32x4 c[S::kChunks / 4];                                 // the next tile's rows, on their way
  float2 f_next;
  int n_rows = per * G;                                    // of a whole tile; `offsets` are set for it
  auto first_of = [&](int i) { return G <= 16 ? i * per : i / parts; };   // (from tok_a on)
  auto load = [&](int i) {
    const int first = first_of(i);
    if (G > 16) {
      const int h0 = (i - first * parts) * 16;
      n_rows = min(16, G - h0);
      offsets(n_rows, h0);
    }
    const char* base = qb + (size_t)first * tok_bytes;
#pragma unroll
    for (int k = 0; k < S::kChunks / 4; ++k) c[k] = *reinterpret_cast<const u32x4*>(base + off[k]);
    f_next = fb[(size_t)first * a.heads + f_off];
    if (r >= n_rows) f_next = make_float2(__builtin_inff(), 0.f);   // (exp2(-inf) * 0)
  };
  auto put = [&]() {
#pragma unroll
    for (int k = 0; k < S::kChunks / 4; ++k)
      *reinterpret_cast<u32x4*>(stage + S::at(S::row(k, lane), S::chunk(k, lane))) = c[k];
    wave_order();
  };
  auto take = [&](uint4 (&q)[terms<E>()][D / 32]) {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      constexpr int kEach = sizeof(E) / 2;                 // chunks of 8 values
      u32x4 v[kEach];
#pragma unroll
      for (int u = 0; u < kEach; ++u)
        v[u] = *reinterpret_cast<const u32x4*>(stage + S::at(r, (g * (D / 32) + ks) * kEach + u));
      if constexpr (sizeof(E) == 2) {
        q[0][ks] = make_uint4(v[0][0], v[0][1], v[0][2], v[0][3]);
      } else {
        const float w[8] = {__uint_as_float(v[0][0]), __uint_as_float(v[0][1]), __uint_as_float(v[0][2]), __uint_as_float(v[0][3]),
                            __uint_as_float(v[1][0]), __uint_as_float(v[1][1]), __uint_as_float(v[1][2]), __uint_as_float(v[1][3])};
        uint4 t[terms<E>()];
        split_terms<terms<E>()>(w, t);
#pragma unroll
        for (int n = 0; n < terms<E>(); ++n) q[n][ks] = t[n];
      }
    }
    wave_order();
  };
  uint4 q[terms<E>()][D / 32];
  if (full < tiles && wave == (full & 3)) {                // the tile that is short of tokens
    n_rows = (toks - full * per) * G;
    offsets(n_rows, 0);
    load(full);
    put();
    take(q);
    add_rows<E, D, true>(x, q, f_next, r < n_rows ? old + tok_a + full * per + my_ti - j0 : -1, acc);
    n_rows = per * G;
  }
  int i = ((full - 1 - wave) & ~3) + wave;                 // (the wave's last whole tile; below 0: it has none)
  if (i >= 0) {
    offsets(n_rows, 0);
    load(i);
    put();
  }
  // a tile's rows leave LDS, the next tile's go there from the registers they came to, and those of the one after set out
  for (; i >= plain; i -= 4) {
    const float2 f = f_next;
    take(q);
    if (i >= 4) load(i - 4);
    add_rows<E, D, false>(x, q, f, 0, acc);
    if (i >= 4) put();
  }
  for (; i >= 0; i -= 4) {
    const float2 f = f_next;
    const int sees = r < n_rows ? old + tok_a + first_of(i) + my_ti - j0 : -1;
    take(q);
    if (i >= 4) load(i - 4);
    add_rows<E, D, true>(x, q, f, sees, acc);
    if (i >= 4) put();
  }
  sums[wave][16 * (r >> 2) + 4 * g + (r & 3)] = sum_rows(acc);
  __syncthreads();
  if (threadIdx.x < kKeyUnit)
    add_mark(sa, rec, x.j0 + threadIdx.x, kvh,
             (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]));
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
// largest, and the kept ones behind place `keep` go to the places of the dropped ones before it, in order.
// No two moves touch one place.  A block's chain of steps bounds it, not the bytes: up to kEvictShort tokens have
// their marks read once, into registers (k_evict); longer sequences go through memory again in each step (k_evict_long).
// Under the profiler: 16 sequences of 8192 tokens and 8 kv heads x 128 down to 512, 24.4 us on 128 of the 256 compute units
// (the blocks of 1024 threads keep 98 scalar registers, of ballots, in vector lanes, which lengthens the chain);
// 40 of 257 down to 256, 8.3 us.
constexpr uint32_t kProtected = 0xffffffffu, kNanKey = 0xfffffffeu;
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return kNanKey;
  const uint32_t u = __float_as_uint(w + 0.f);             // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr int kBins = 2048;
constexpr int kEvictShort = 16 * 1024, kPageCache = kEvictShort / 16;

// From `hist`, counts of digits: the digit that the `need`-th largest key has, and its rank among those.  All threads
// call it; kWaves waves, whose totals are in `wave`.
template <int kWaves>
__device__ __forceinline__ void find_digit(const uint32_t* hist, uint32_t* wave, uint32_t* found, int need) {
  constexpr int kEach = kBins / (64 * kWaves);             // bins of a lane, the largest digits in the first lane
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint32_t c[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += c[i] = hist[kBins - 1 - (tid * kEach + i)];
  uint32_t upto = sum;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const uint32_t o = __shfl_up(upto, i);
    upto += lane >= i ? o : 0u;
  }
  if (lane == 63) wave[wv] = upto;
  __syncthreads();
  uint32_t before = upto - sum;
  for (int i = 0; i < wv; ++i) before += wave[i];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (before < (uint32_t)need && before + c[i] >= (uint32_t)need) {
      found[0] = kBins - 1 - (tid * kEach + i);
      found[1] = (uint32_t)need - before;
    }
    before += c[i];
  }
  __syncthreads();
}

struct alignas(16) EvictLds {
  union {
    uint32_t hist[kBins];
    uint32_t count[kEvictShort / 64];                      // of each 64 places
  };
  uint32_t wave[16], found[2];
  int32_t newest;
  uint16_t hole[kEvictShort / 2], mover[kEvictShort / 2];
};

template <int NT, int IT>   // threads, tokens of each
__global__ void __launch_bounds__(NT) k_evict(EvictArgs a) {
  constexpr int kItems = IT;
  __shared__ EvictLds sh;
  __shared__ int32_t s_page[kPageCache];
  constexpr int kWaves = NT / 64, kWords = kItems * kWaves;
  const int seq = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  const SeqRec rec = a.b.rec[seq];
  const int n = rec.len, keep = a.keep, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (n <= keep) return;
  const int lp = a.kv.log2_page, hk = a.kv.kv_heads;
  for (int i = tid; i <= (n - 1) >> lp; i += NT) s_page[i] = a.b.pages[rec.ref0 + i];
  if (tid == 0) sh.newest = INT32_MIN;
  for (int i = tid; i < kBins; i += NT) sh.hist[i] = 0;
  __syncthreads();
  auto vec_of = [&](int j) { return (((size_t)s_page[j >> lp] * hk + kvh) << lp) + (j & ((1 << lp) - 1)); };
  // token it * NT + tid in item `it`: a wave has 64 places in a row
  uint32_t key[kItems];
  {
    float w[kItems];
    int p[kItems];
    int top = INT32_MIN;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const size_t v = vec_of(min(it * NT + tid, n - 1));  // (past the last token: that one again)
      w[it] = a.kv.weight[v];
      p[it] = a.kv.place[v];
    }
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      top = max(top, p[it]);
    }
    for (int i = 1; i < 64; i *= 2) top = max(top, __shfl_xor(top, i));
    if (lane == 0) atomicMax(&sh.newest, top);
    __syncthreads();
    const int64_t since = (int64_t)sh.newest - a.recent;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      key[it] = a.recent > 0 && (int64_t)p[it] > since ? kProtected : weight_order(w[it]);
    }
  }
  // the keep-th largest key: `prefix`, of which `need` stay
  uint32_t prefix = 0;
  int need = keep;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      if (it * NT + tid < n && (pass == 0 || (key[it] >> (shift + width)) == (prefix >> (shift + width))))
        atomicAdd(&sh.hist[(key[it] >> shift) & ((1u << width) - 1u)], 1u);
    }
    __syncthreads();
    find_digit<kWaves>(sh.hist, sh.wave, sh.found, need);
    prefix |= sh.found[0] << shift;
    need = (int)sh.found[1];
    for (int i = tid; i < kBins; i += NT) sh.hist[i] = 0;
    __syncthreads();
  }
  // Sums over the 64-place words before each word, in order: by wave 0, whose lanes have kWords / 64 words each.
  auto scan = [&]() {
    __syncthreads();
    if (wv == 0) {
      constexpr int kEach = (kWords + 63) / 64;
      uint32_t c[kEach], sum = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) sum += c[i] = lane * kEach + i < kWords ? sh.count[lane * kEach + i] : 0u;
      uint32_t upto = sum;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        const uint32_t o = __shfl_up(upto, i);
        upto += lane >= i ? o : 0u;
      }
      uint32_t before = upto - sum;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (lane * kEach + i < kWords) sh.count[lane * kEach + i] = before;
        before += c[i];
      }
      if (lane == 63) sh.found[0] = before;
    }
    __syncthreads();
  };
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    const uint64_t same = __ballot(it * NT + tid < n && key[it] == prefix);
    if (lane == 0) sh.count[it * kWaves + wv] = (uint32_t)__popcll(same);
  }
  scan();
  uint32_t stays = 0;                                      // bit `it`
  uint32_t mine[kItems];                                   // holes in the lower half, movers in the upper one
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    const int j = it * NT + tid;
    const uint64_t same = __ballot(j < n && key[it] == prefix);
    const int rank = (int)sh.count[it * kWaves + wv] + __popcll(same & below);
    const bool s = j < n && (key[it] > prefix || (key[it] == prefix && rank < need));
    stays |= (uint32_t)s << it;
    mine[it] = (uint32_t)__popcll(__ballot(j < keep && !s)) | ((uint32_t)__popcll(__ballot(j >= keep && s)) << 16);
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    if (lane == 0) sh.count[it * kWaves + wv] = mine[it];
  }
  scan();
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    const int j = it * NT + tid;
    const bool s = (stays >> it) & 1;
    const uint32_t before = sh.count[it * kWaves + wv];
    const uint64_t hs = __ballot(j < keep && !s), ms = __ballot(j >= keep && s);
    if (j < keep && !s) sh.hole[(before & 0xffffu) + __popcll(hs & below)] = (uint16_t)j;
    if (j >= keep && s) sh.mover[(before >> 16) + __popcll(ms & below)] = (uint16_t)j;
  }
  __syncthreads();
  const int total = (int)(sh.found[0] & 0xffffu), dv = a.kv.dim / 16;   // (as many movers)
  const int log_dv = 31 - __builtin_clz(dv);
  for (int i0 = tid; i0 < total * 2 * dv; i0 += 4 * NT) {
    u32x4 c[4];
    uint8_t* to[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * NT;
      if (i >= total * 2 * dv) continue;
      const int mv = i >> (log_dv + 1), part = i & (2 * dv - 1);
      uint8_t* p = part < dv ? a.kv.k : a.kv.v;
      const int o = (part & (dv - 1)) * 16;
      c[u] = *reinterpret_cast<const u32x4*>(p + vec_of(sh.mover[mv]) * a.kv.dim + o);
      to[u] = p + vec_of(sh.hole[mv]) * a.kv.dim + o;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * NT < total * 2 * dv) *reinterpret_cast<u32x4*>(to[u]) = c[u];
  }
  for (int i = tid; i < total; i += NT) {
    const size_t from = vec_of(sh.mover[i]), to = vec_of(sh.hole[i]);
    const float ks = a.kv.ks[from], vs = a.kv.vs[from], w = a.kv.weight[from];
    const int p = a.kv.place[from];
    a.kv.ks[to] = ks;
    a.kv.vs[to] = vs;
    a.kv.weight[to] = w;
    a.kv.place[to] = p;
  }
}

// The same for longer sequences: a bit for each token in LDS says which stay, and moves are listed kMoves at a time, each
// list by going through all bits again.  Two sequences of 131072 tokens and 8 kv heads x 128 down to 4096: 489 us; one
// head of 2^19 down to 2^18, 131072 moves, 11.5 ms.
constexpr int kMoves = 2048;
struct alignas(16) EvictLongLds {                          // dynamic LDS: these, and the bits
  uint32_t hist[kBins];
  int32_t hole[kMoves], mover[kMoves];
  int32_t wave[16], wave2[16];
  uint32_t digits[16], found[2];
  int32_t newest;
};

__global__ void __launch_bounds__(1024) k_evict_long(EvictArgs a) {
  constexpr int NT = 1024;
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  EvictLongLds& sh = *reinterpret_cast<EvictLongLds*>(dyn);
  uint32_t* bits = reinterpret_cast<uint32_t*>(dyn + sizeof(EvictLongLds));
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
  auto key_of = [&](int j) {
    const size_t v = vec_of(j);
    const uint32_t k = weight_order(a.kv.weight[v]);
    return a.recent > 0 && (int64_t)a.kv.place[v] > since ? kProtected : k;
  };
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
    find_digit<kWaves>(sh.hist, sh.digits, sh.found, need);
    prefix |= sh.found[0] << shift;
    need = (int)sh.found[1];
    __syncthreads();
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
  if (a.n_joins && sa.many)
    hipLaunchKernelGGL(k_score_join, dim3((unsigned)(((int64_t)a.n_joins * a.heads + 15) / 16)), dim3(256), 0, s, sa);
  const int units = sa.b.n_units;
  if (units && sa.many)
    hipLaunchKernelGGL((k_score_many<E, D, FMT>), dim3((unsigned)score_blocks(units, a.kv.kv_heads)), dim3(256), 0, s, sa);
  if (units && sa.few)
    hipLaunchKernelGGL((k_score_few<E, D, FMT>), dim3((unsigned)score_blocks((units + 3) / 4, a.kv.kv_heads)), dim3(256), 0, s,
                       sa);
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
  const dim3 grid((unsigned)((int64_t)a.b.n_seqs * a.kv.kv_heads));
  if (a.max_len <= 1024) hipLaunchKernelGGL((k_evict<256, 4>), grid, dim3(256), 0, s, a);
  else if (a.max_len <= 4096) hipLaunchKernelGGL((k_evict<512, 8>), grid, dim3(512), 0, s, a);
  else if (a.max_len <= kEvictShort) hipLaunchKernelGGL((k_evict<1024, 16>), grid, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL(k_evict_long, grid, dim3(1024), (int)sizeof(EvictLongLds) + (a.max_len + 63) / 64 * 8, s, a);
  return hipGetLastError();
}

}  // namespace salt
