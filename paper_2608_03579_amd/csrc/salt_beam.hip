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
// The value of the lane below (lane 0: 0).
__device__ __forceinline__ uint32_t from_below(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x138, 0xf, 0xf, true);   // wave_shr:1
}
__device__ __forceinline__ uint64_t from_below(uint64_t v) {
  return ((uint64_t)from_below((uint32_t)(v >> 32)) << 32) | from_below((uint32_t)v);
}

// The best n entries so far, the i-th best in lane i; 0 where there are fewer.
struct Best {
  uint64_t e = 0, least = 0;                               // least: the n-th
  // `v` (the same in all lanes) goes to its place; the entries behind move up a lane.
  __device__ __forceinline__ void insert(uint64_t v, int n) {
    const int at = __popcll(__ballot(e > v)), lane = threadIdx.x & 63;
    const uint64_t up = from_below(e);
    e = lane < at ? e : lane == at ? v : up;
    const uint64_t last = lane_value(e, n - 1);
    least = last > least ? last : least;
  }
  // One entry of every lane.
  __device__ __forceinline__ void offer(uint64_t v, int n) {
    uint64_t who = __ballot(v > least);
    while (who) {
      insert(lane_value(v, __builtin_ctzll(who)), n);
      who &= who - 1;
      who &= __ballot(v > least);
    }
  }
};
// A number that the n-th largest of the lanes' keys is not below: its upper 16 bits.  (0: fewer than n lanes have one)
__device__ __forceinline__ uint32_t nth_at_least(uint32_t key, int n) {
  uint32_t t = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t c = t | (1u << bit);
    if (__popcll(__ballot(key >= c)) >= n) t = c;
  }
  return t;
}

__device__ __forceinline__ float largest(const float (&v)[16]) {
  float top = max3_of(v[0], v[1], v[2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) top = max3_of(top, v[i], v[i + 1]);
  return max3_of(top, v[15], v[15]);
}

// One piece of one row: a block of four waves, which take runs of 1024 logits in turn, 16 to a lane.  A lane's
// maximum decides whether its logits are looked at, and the waves tell each other bounds, so that few of them enter a
// list only to leave it.  512 rows of 128256 logits in bf16, 16 continuations: 45 us under the profiler (2.9
// TB/s), in fp32 48 (5.5 TB/s).  Of the 45 the vector unit is busy for 27 (225 instructions to a run, 16 of them exponentials)
// and the bytes take 25 at a copy's rate: neither bounds it, they overlap badly.  Lists entered value by
// value took 157 us, by ballot 56, with bounds between waves 45; twice or half as many blocks to a row 52.  Four rows:
// 8 us, a chain of launch, load and list.
constexpr int kRun = 1024;
template <typename E>
__global__ void __launch_bounds__(256) k_beam_scan(BeamArgs a) {
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.n_out;
  const int runs = (a.vocab + kRun - 1) / kRun;
  const int c0 = (int)((int64_t)runs * split / a.splits), c1 = (int)((int64_t)runs * (split + 1) / a.splits);
  const E* x = reinterpret_cast<const E*>(a.logits) + (int64_t)row * a.ld;
  Best best;
  float m = kNegInf;
  double sum = 0.;
  using Vec = typename Ops<E>::Vec;
  // (the last run's end, value by value: nothing behind the vocabulary is read)
  auto load = [&](int c, Vec (&v)[2]) {
    const int at = c * kRun + lane * 8;
    if ((c + 1) * kRun <= a.vocab) {
      v[0] = Ops<E>::load(x + at);
      v[1] = Ops<E>::load(x + at + 512);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t w[Ops<E>::kWords];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = at + 512 * u + i;
          if constexpr (sizeof(E) == 4) {
            w[i] = k < a.vocab ? __float_as_uint(x[k]) : 0xff800000u;
          } else {
            const uint32_t b = k < a.vocab ? x[k] : 0xff80u;
            w[i / 2] = i & 1 ? w[i / 2] | (b << 16) : b;
          }
        }
        v[u] = Ops<E>::vec(w);
      }
    }
  };
  Vec raw[2], next[2], after[2];                           // (two runs on their way while one is worked on)
  int c = c0 + wave;
  if (c < c1) load(c, raw);
  if (c + 4 < c1) load(c + 4, next);
  // A bound of the block's n-th best: where each wave has n / 4 keys that are not below t, n of the block are not.  From
  // the lanes' maxima to begin with, then from the waves' lists as they stand (keys only grow, an older one is a bound, too).
  __shared__ uint32_t s_key[4];
  const int quarter = (n + 3) / 4;
  {
    uint32_t most = 0;
    if (c < c1) {
      float v[16];
      Ops<E>::to_f32(raw[0], v);
      Ops<E>::to_f32(raw[1], v + 8);
      most = order_of(largest(v));
    }
    const uint32_t t = nth_at_least(most, n);
    best.least = t ? entry_of(t - 1, 0) : 0;               // (entries of the key t itself are above it)
    if (lane == 0) s_key[wave] = nth_at_least(most, quarter);
    __syncthreads();
  }
  auto key_of_wave = [&](int w) { return __hip_atomic_load(&s_key[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); };
  for (; c < c1; c += 4) {
    if (c + 8 < c1) load(c + 8, after);
    const uint32_t t = min(min(key_of_wave(0), key_of_wave(1)), min(key_of_wave(2), key_of_wave(3)));
    const uint64_t bound = t ? entry_of(t - 1, 0) : 0;
    float v[16];
    Ops<E>::to_f32(raw[0], v);
    Ops<E>::to_f32(raw[1], v + 8);
    // the sum of exponentials under the lane's own maximum
    const float top = largest(v);
    if (top > m) {
      if (m > kNegInf) sum *= (double)__builtin_amdgcn_exp2f((m - top) * kLog2e);
      m = top;
    }
    const float mu = m == kNegInf ? 0.f : m;
    float part[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) part[i & 1] += __builtin_amdgcn_exp2f((v[i] - mu) * kLog2e);
    sum += (double)(part[0] + part[1]);
    // (NaNs pass unseen: their row offers nothing in the end)
    const uint32_t most = order_of(top);
    best.least = bound > best.least ? bound : best.least;
    if (__any(most && entry_of(most, 0) > best.least)) {
      // (a value that can enter is not below the n-th best's; entries decide among equals)
      const float bar = value_of(max((uint32_t)(best.least >> 32), 0x00800000u));
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (__any(v[i] >= bar)) {
          const uint32_t key = order_of(v[i]);
          best.offer(key ? entry_of(key, (uint32_t)(c * kRun + (i >> 3) * 512 + lane * 8 + (i & 7))) : 0, n);
        }
      const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)(best.e >> 32), quarter - 1);
      if (lane == 0 && mine > key_of_wave(wave)) __hip_atomic_store(&s_key[wave], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) raw[u] = next[u], next[u] = after[u];
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
    if (at < n) a.best[((int64_t)row * n + at) * a.splits + split] = e;
  }
  if (threadIdx.x == 0) {
    const float mm = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    double t = 0.;
    for (int i = 0; i < 4; ++i)
      t += s_m[i] > kNegInf ? s_sum[i] * (double)__builtin_amdgcn_exp2f((s_m[i] - mm) * kLog2e) : s_sum[i];
    a.stat[piece] = make_double2((double)mm, t);
  }
}

// Doubles as numbers of the same order.
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.);
  return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}

// One request.  A wave joins the pieces of a beam (their best first, so that few of the others enter the list), and
// enters that list, by worth, into one for all beams it takes; the place of an entry of the waves' lists
// is then the number of better ones.
constexpr int kJoinWaves = 8;
struct Worth {
  uint64_t w = 0;                                          // order of the worth; 0: none
  uint32_t beam = 0, token = 0;
};
__global__ void __launch_bounds__(64 * kJoinWaves) k_beam_join(BeamArgs a) {
  const int req = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.n_out;
  __shared__ uint64_t s_w[kJoinWaves * kMaxOut];
  __shared__ uint32_t s_beam[kJoinWaves * kMaxOut];
  Worth all;
  for (int b = wave; b < a.width; b += kJoinWaves) {
    const int64_t row = (int64_t)req * a.width + b;
    const uint64_t* lists = a.best + row * n * a.splits;
    const int total = n * a.splits;
    uint64_t e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) e[u] = u * 64 + lane < total ? lists[u * 64 + lane] : 0;
    double2 st = make_double2(-__builtin_inf(), 0.);
    if (lane < a.splits) st = a.stat[row * a.splits + lane];
    const float score = a.score[row];
    double m = st.x;
    for (int i = 1; i < a.splits; i *= 2) m = fmax(m, __shfl_xor(m, i));
    double sum = st.x > -__builtin_inf() ? st.y * exp(st.x - m) : st.y;
    for (int i = 1; i < a.splits; i *= 2) sum += __shfl_xor(sum, i);
    // (a row with a NaN or +inf has a sum of NaN, one without a logit above -inf a sum of 0; lane 0 has the row's own)
    if (!__builtin_amdgcn_readfirstlane((int)(score > kNegInf && score < __builtin_inff() && sum > 0.))) continue;
    const double mine = (double)score - (m + log(sum));
    const double c = __builtin_bit_cast(double, lane_value(__builtin_bit_cast(uint64_t, mine), 0));
    Best best;
    if (a.splits == 1) {
      best.e = e[0];
    } else {
      const uint32_t t = nth_at_least((uint32_t)(e[0] >> 32), n);
      best.least = t ? entry_of(t - 1, 0) : 0;
      for (int first = 0; first < total; first += 256) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint64_t now = e[u];
          const int at = first + 256 + u * 64 + lane;
          e[u] = at < total ? lists[at] : 0;
          best.offer(now, n);
        }
      }
    }
    Worth x;
    if (lane < n && best.e)
      x = Worth{order_of((double)value_of((uint32_t)(best.e >> 32)) + c), (uint32_t)b, ~(uint32_t)best.e};
    if (b == wave) {
      all = x;
      continue;
    }
    // (in order; equal worth: the beams before this one go first)
    for (int i = 0; i < n; ++i) {
      const uint64_t v = lane_value(x.w, i);
      const int at = __popcll(__ballot(all.w >= v));
      if (v == 0 || at >= n) break;
      const uint32_t tok = (uint32_t)__builtin_amdgcn_readlane((int)x.token, i);
      const uint64_t wu = from_below(all.w);
      const uint32_t bu = from_below(all.beam), tu = from_below(all.token);
      if (lane == at) all = Worth{v, (uint32_t)b, tok};
      else if (lane > at) all = Worth{wu, bu, tu};
    }
  }
  const int at = wave * n + lane;
  if (lane < n) s_w[at] = all.w, s_beam[at] = all.beam;
  __syncthreads();
  const int total = min(a.width, kJoinWaves) * n;
  if (lane >= n || at >= total) return;
  int better = 0;
#pragma unroll 8
  for (int i = 0; i < total; ++i) {
    const uint64_t w = s_w[i];
    const uint32_t b = s_beam[i];
    better += (int)(w > all.w) | ((int)(w == all.w) & ((int)(b < all.beam) | ((int)(b == all.beam) & (int)(i < at))));
  }
  if (better >= n) return;
  const int64_t to = (int64_t)req * n + better;
  const double w = __builtin_bit_cast(double, all.w >> 63 ? all.w ^ ((uint64_t)1 << 63) : ~all.w);
  a.out_score[to] = all.w ? (float)w : kNegInf;
  a.out_beam[to] = all.w ? (int)all.beam : -1;
  a.out_token[to] = all.w ? (int)all.token : -1;
}

// A block takes one kv head of one page in one layer.  128 pages, half full, in 28 layers of 8 heads x 128: 492 MB in
// and out in 118 us, 4.2 TB/s.
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
  hipLaunchKernelGGL(k_beam_join, dim3(a.reqs), dim3(64 * kJoinWaves), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_copy_pages, dim3(a.n * a.kv.kv_heads, a.n_layers), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace salt
