// The base product of a table in 8 bits: y = x W_base, which the apply then adds to.
// W and x are held as e4m3 codes with one fp32 scale for each block of 128 inputs x
// 128 outputs (W) and of 128 inputs (x, per token):
//
//   s = max(amax * (1/448), 2^-126),  code = e4m3(v * (1 / s))       (fp32, rounded to nearest even)
//   y[t][o] = rnd( sum_kb  s_x[t][kb] s_w[kb][o / 128]  sum_{k in kb} xq[t][k] wq[k][o] )
//
// The inner sum over 128 inputs is one matrix instruction (16x16x128, fp32
// accumulation); its result times the two scales is added to the fp32 total, so the
// scales may be any fp32 values.  e4m3 keeps a relative error of 2^-4 per value: the
// two roundings to codes are the only ones before y's own.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "salt_base_rule.h"
#include "salt_device.h"
#include "salt_layout.h"
#include "salt_serve.h"

namespace salt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
constexpr float kE4m3Max = 448.f;

// Scale of a block whose largest magnitude is amax, a number or infinity: with an infinite
// scale every code times it is NaN.  (A NaN in x does not show in amax; its NaN code is enough for its token.)
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(amax * (1.0f / kE4m3Max), 0x1p-126f); }

// Four codes of v * r, first in the lowest byte.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ float e4m3_at(uint32_t w, int i) {
  switch (i & 3) {
    case 0: return __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
}

// An operand of a 16 x 16 x 128 step: lane l holds 32 codes of row (l & 15).
//
// bf16 contexts multiply the codes as they are, in one instruction.  It adds its 128
// products with some 14 bits behind the largest one: 1.4e-5 of a result's size (2048
// random inputs), a hundredth of y's own rounding.  fp32 contexts take the codes to
// bf16, where they are exact, and four instructions that add in fp32 (4.7e-8), at half
// the rate.
template <typename E>
struct Codes;
template <>
struct Codes<uint16_t> {
  i32x8 v;
  __device__ __forceinline__ void set(const i32x8& c) { v = c; }
  // a b^T from zero: lane l receives column (l & 15), rows 4 (l >> 4) .. + 3.
  // (Constant zeros for the instruction's own scales select the form without them.)
  static __device__ __forceinline__ f32x4 mma(const Codes& a, const Codes& b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <>
struct Codes<float> {
  uint4 v[4];
  __device__ __forceinline__ void set(const i32x8& c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = __builtin_bit_cast(uint32_t, (q & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j + (q >> 1)], 1.0f, true)
                                                    : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * j + (q >> 1)], 1.0f, false));
      v[j] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  static __device__ __forceinline__ f32x4 mma(const Codes& a, const Codes& b) {
    f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = Ops<uint16_t>::mma(a.v[j], b.v[j], c);
    return c;
  }
};
__device__ __forceinline__ i32x8 load_tile(const uint8_t* tile, int lane) {
  const uint4 a = *reinterpret_cast<const uint4*>(tile + lane * 16);
  const uint4 b = *reinterpret_cast<const uint4*>(tile + 1024 + lane * 16);
  return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// Output of row `r` of tile `t` (salt_serve.h), and back: its tile and row.
__host__ __device__ constexpr int out_of(int t, int r) { return 32 * (t >> 1) + 8 * (r >> 2) + 4 * (t & 1) + (r & 3); }
__host__ __device__ constexpr int tile_of(int o) { return 2 * (o >> 5) + ((o >> 2) & 1); }
__host__ __device__ constexpr int row_of(int o) { return 4 * ((o >> 3) & 3) + (o & 3); }

// ---------------------------------------------------------------------------
// weights in and out (once at start-up: simple kernels, one block per 128 x 128)
// ---------------------------------------------------------------------------
constexpr int kPinLd = kBaseBlock + 4;

// The block of codes in s_q ([output][input], kPinLd bytes apart) to its 8 tiles.
__device__ __forceinline__ void store_block(const BasePinArgs& a, const uint8_t* s_q, int kb, int nb) {
  for (int p = threadIdx.x; p < 8 * 2 * 64; p += 256) {
    const int t = p >> 7, h = (p >> 6) & 1, l = p & 63;
    const int o = out_of(t, l & 15), k = 32 * (l >> 4) + 16 * h;
    const uint32_t* q = reinterpret_cast<const uint32_t*>(s_q + o * kPinLd + k);
    *reinterpret_cast<uint4*>(a.tab.w + ((size_t)(nb * 8 + t) * a.kb + kb) * kBaseTile + h * 1024 + l * 16) =
        make_uint4(q[0], q[1], q[2], q[3]);
  }
}

template <typename E>
__global__ void __launch_bounds__(256) k_base_pin(BasePinArgs a) {
  __shared__ float s_v[kBaseBlock][kBaseBlock + 1];   // [input][output]
  __shared__ __attribute__((aligned(16))) uint8_t s_q[kBaseBlock * kPinLd];
  __shared__ uint32_t s_max[4];
  const int kb = blockIdx.x, nb = blockIdx.y, tid = threadIdx.x;
  // the bits of the magnitudes order like the magnitudes, NaN above infinity
  uint32_t amax = 0;
  for (int p = tid; p < kBaseBlock * (kBaseBlock / 8); p += 256) {
    const int k = p >> 4, o = (p & 15) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (kb * kBaseBlock + k < a.in && nb * kBaseBlock + o < a.tab.out)
      Ops<E>::to_f32(Ops<E>::load(reinterpret_cast<const E*>(a.w) + (size_t)(kb * kBaseBlock + k) * a.ld +
                                  nb * kBaseBlock + o), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s_v[k][o + e] = v[e];
      amax = max(amax, __float_as_uint(v[e]) & 0x7fffffffu);
    }
  }
  for (int m = 1; m < 64; m *= 2) amax = max(amax, (uint32_t)__shfl_xor((int)amax, m));
  if ((tid & 63) == 0) s_max[tid >> 6] = amax;
  __syncthreads();
  const float top = __uint_as_float(max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3])));
  const float s = top == top ? block_scale(top) : top;     // (a NaN takes the block, as an infinity does)
  const float r = 1.0f / s;
  for (int p = tid; p < kBaseBlock * (kBaseBlock / 4); p += 256) {
    const int o = p & 127, k = (p >> 7) * 4;
    *reinterpret_cast<uint32_t*>(s_q + o * kPinLd + k) =
        pack_e4m3(s_v[k][o] * r, s_v[k + 1][o] * r, s_v[k + 2][o] * r, s_v[k + 3][o] * r);
  }
  if (tid == 0) a.tab.sw[(size_t)kb * a.tab.n_blk + nb] = s;
  __syncthreads();
  store_block(a, s_q, kb, nb);
}

__global__ void __launch_bounds__(256) k_base_pin_codes(BasePinArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t s_q[kBaseBlock * kPinLd];
  const int kb = blockIdx.x, nb = blockIdx.y, tid = threadIdx.x;
  for (int p = tid; p < kBaseBlock * (kBaseBlock / 8); p += 256) {
    const int o = p >> 4, k = (p & 15) * 8;
    uint2 v = make_uint2(0u, 0u);
    if (nb * kBaseBlock + o < a.tab.out && kb * kBaseBlock + k < a.in)
      v = *reinterpret_cast<const uint2*>(a.q + (size_t)(nb * kBaseBlock + o) * a.ld + kb * kBaseBlock + k);
    *reinterpret_cast<uint32_t*>(s_q + o * kPinLd + k) = v.x;
    *reinterpret_cast<uint32_t*>(s_q + o * kPinLd + k + 4) = v.y;
  }
  // (blocks of the padding have no scale of their own)
  if (tid == 0)
    a.tab.sw[(size_t)kb * a.tab.n_blk + nb] = nb * kBaseBlock < a.tab.out ? a.sq[(size_t)nb * a.kb + kb] : 0.f;
  __syncthreads();
  store_block(a, s_q, kb, nb);
}

template <typename E>
__global__ void __launch_bounds__(256) k_base_read(BasePinArgs a) {
  const int kb = blockIdx.x, nb = blockIdx.y;
  const float s = a.tab.sw[(size_t)kb * a.tab.n_blk + nb];
  for (int p = threadIdx.x; p < kBaseBlock * (kBaseBlock / 8); p += 256) {
    const int k = p >> 4, o8 = (p & 15) * 8, gk = kb * kBaseBlock + k, go = nb * kBaseBlock + o8;
    if (gk >= a.in || go >= a.tab.out) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int o = go + e;
      const uint8_t* t = a.tab.w + ((size_t)tile_of(o) * a.kb + kb) * kBaseTile;
      const int lane = 16 * (k >> 5) + row_of(o);
      v[e] = e4m3_at(t[((k >> 4) & 1) * 1024 + lane * 16 + (k & 15)], 0) * s;
    }
    Ops<E>::store(reinterpret_cast<E*>(a.w) + (size_t)gk * a.ld + go, v);
  }
}

// ---------------------------------------------------------------------------
// x to codes
// ---------------------------------------------------------------------------
// One wave per 16 tokens x 128 inputs: lane l holds 32 inputs of token (l & 15), the
// four lanes of a token share the block's largest magnitude.  Inputs past `in` are
// zeros; tokens past T repeat the last one (their codes are never stored to y).
template <typename E>
__device__ __forceinline__ i32x8 quantise_x(const E* x, int T, int in, int tile, int kb, int lane, float& scale) {
  using O = Ops<E>;
  const int t = min(16 * tile + (lane & 15), T - 1), k0 = kb * kBaseBlock + 32 * (lane >> 4);
  float v[32];
  const E* row = x + (size_t)t * in;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const typename O::Vec w = k0 + 8 * j < in ? O::load(row + k0 + 8 * j) : O::zero();
    O::to_f32(w, v + 8 * j);
  }
  float amax = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) amax = fmaxf(amax, fabsf(v[e]));
  amax = fmaxf(amax, __shfl_xor(amax, 16));
  amax = fmaxf(amax, __shfl_xor(amax, 32));
  scale = block_scale(amax);
  const float r = 1.0f / scale;
  i32x8 q;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    q[j] = (int)pack_e4m3(v[4 * j] * r, v[4 * j + 1] * r, v[4 * j + 2] * r, v[4 * j + 3] * r);
  return q;
}

template <typename E>
__global__ void __launch_bounds__(256) k_base_quantise(BaseArgs a) {
  const int lane = threadIdx.x & 63, tile = blockIdx.x, kb = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (kb >= a.kb) return;
  float s;
  const i32x8 q = quantise_x(reinterpret_cast<const E*>(a.x), a.T, a.in, tile, kb, lane, s);
  uint8_t* t = a.xq + ((size_t)tile * a.kb + kb) * kBaseTile;
  *reinterpret_cast<uint4*>(t + lane * 16) = make_uint4(q[0], q[1], q[2], q[3]);
  *reinterpret_cast<uint4*>(t + 1024 + lane * 16) = make_uint4(q[4], q[5], q[6], q[7]);
  if (lane < 16) a.sx[(size_t)kb * a.T_pad + 16 * tile + lane] = s;
}

// ---------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------
__device__ __forceinline__ void store8(uint16_t* p, const f32x4& lo, const f32x4& hi) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]),
                                            pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3]));
}
__device__ __forceinline__ void store8(float* p, const f32x4& lo, const f32x4& hi) {
  *reinterpret_cast<float4*>(p) = make_float4(lo[0], lo[1], lo[2], lo[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(hi[0], hi[1], hi[2], hi[3]);
}

// The table of work item `i` of the launch (items of a table stand together).
__device__ __forceinline__ int table_of(const BaseArgs& a, int i) {
  int t = 0;
  while (t + 1 < a.n_tables && i >= a.tab[t + 1].first) ++t;
  return t;
}

// acc += p * s, a block of 128 inputs' products times its two scales.
__device__ __forceinline__ void add_scaled(f32x4& acc, const f32x4& p, float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], s, acc[e]);
}

// Up to 16 tokens, in one launch: a block takes OT (1 or 2) tiles of 16 outputs, its 16 waves the
// input blocks in turn; each wave quantises the x it multiplies (16 tokens x 128 inputs,
// read from L2 by every block), and the waves' sums meet in LDS.  One token: 3072 x 3072 4.5 us, a
// launch's own time and two memory latencies; 28672 x 4096 25 us, 4.7 TB/s of weights.
constexpr int kFewWaves = 16;
template <typename E, int OT>
__global__ void __launch_bounds__(64 * kFewWaves) k_base_few(BaseArgs a) {
  __shared__ __attribute__((aligned(16))) f32x4 s_acc[OT][kFewWaves][64];
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BaseTable& tab = a.tab[table_of(a, blockIdx.x)];
  const int tile = (blockIdx.x - tab.first) * OT;
  const size_t row = (size_t)a.kb * kBaseTile;
  const uint8_t* w = tab.w + tile * row;
  const float* sw = tab.sw + tile / 8;
  f32x4 acc[OT];
#pragma unroll
  for (int i = 0; i < OT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = wave; kb < a.kb; kb += 2 * kFewWaves) {
    // two blocks' weights on their way before either is used
    const bool two = kb + kFewWaves < a.kb;
    const int kb2 = two ? kb + kFewWaves : kb;
    i32x8 w0[OT], w1[OT];
#pragma unroll
    for (int i = 0; i < OT; ++i) {
      w0[i] = load_tile(w + i * row + (size_t)kb * kBaseTile, lane);
      w1[i] = load_tile(w + i * row + (size_t)kb2 * kBaseTile, lane);
    }
    const float s0 = sw[(size_t)kb * tab.n_blk], s1 = sw[(size_t)kb2 * tab.n_blk];
    Codes<E> cw, cx;
    float sx;
    cx.set(quantise_x(reinterpret_cast<const E*>(a.x), a.T, a.in, 0, kb, lane, sx));
#pragma unroll
    for (int i = 0; i < OT; ++i) {
      cw.set(w0[i]);
      add_scaled(acc[i], Codes<E>::mma(cw, cx), s0 * sx);
    }
    if (two) {
      cx.set(quantise_x(reinterpret_cast<const E*>(a.x), a.T, a.in, 0, kb2, lane, sx));
#pragma unroll
      for (int i = 0; i < OT; ++i) {
        cw.set(w1[i]);
        add_scaled(acc[i], Codes<E>::mma(cw, cx), s1 * sx);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < OT; ++i) s_acc[i][wave][lane] = acc[i];
  __syncthreads();
  if (wave >= OT) return;
  f32x4 v = s_acc[wave][0][lane];
#pragma unroll
  for (int q = 1; q < kFewWaves; ++q) v += s_acc[wave][q][lane];
  const int t = lane & 15, o = out_of(tile + wave, 4 * g);
  if (t < a.T && o < tab.out) {
    E* y = reinterpret_cast<E*>(tab.y) + (size_t)t * tab.out + o;
    if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(y) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

// The products of a block's wave tiles to y: token (lane & 15) of token tile j, outputs
// 8 (lane >> 4) .. + 7 of the tile pair.
template <typename E>
__device__ __forceinline__ void store_pair(const BaseArgs& a, const BaseTable& tab, int t0, int o0, int lane,
                                           const f32x4& lo, const f32x4& hi) {
  const int t = t0 + (lane & 15), o = o0 + 8 * (lane >> 4);
  if (t < a.T && o < tab.out) store8(reinterpret_cast<E*>(tab.y) + (size_t)t * tab.out + o, lo, hi);
}

// Batches too small to fill the device with whole products: a block takes OT output tiles x
// TT token tiles, its 8 waves the input blocks in turn, operands straight from L2; the
// waves' sums meet in LDS, where each wave adds up its share of them.  Latency and L2 bound it: 6144
// x 4096 of 64 tokens 7.8 us (26 MB, 3.4 TB/s), 4096 x 4096 of 256 11 us, and 3 for the quantiser.
constexpr int kSplitWaves = 8;
constexpr size_t split_lds(int ot, int tt) { return (size_t)kSplitWaves * ot * tt * 1024; }
template <typename E, int OT, int TT>
__global__ void __launch_bounds__(64 * kSplitWaves) k_base_split(BaseArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  f32x4* s_acc = reinterpret_cast<f32x4*>(lds);        // [tile pair][wave][2][64]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BaseTable& tab = a.tab[table_of(a, blockIdx.x)];
  const int ot0 = (blockIdx.x - tab.first) * OT, tt0 = blockIdx.y * TT;
  f32x4 acc[OT][TT];
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = wave; kb < a.kb; kb += kSplitWaves) {
    Codes<E> w[OT], x[TT];
    float s[TT];
    const float sw = tab.sw[(size_t)kb * tab.n_blk + ot0 / 8];
#pragma unroll
    for (int i = 0; i < OT; ++i) w[i].set(load_tile(tab.w + ((size_t)(ot0 + i) * a.kb + kb) * kBaseTile, lane));
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      x[j].set(load_tile(a.xq + ((size_t)(tt0 + j) * a.kb + kb) * kBaseTile, lane));
      s[j] = a.sx[(size_t)kb * a.T_pad + 16 * (tt0 + j) + (lane & 15)];
    }
#pragma unroll
    for (int j = 0; j < TT; ++j)
#pragma unroll
      for (int i = 0; i < OT; ++i) add_scaled(acc[i][j], Codes<E>::mma(w[i], x[j]), sw * s[j]);
  }
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) s_acc[((((i >> 1) * TT + j) * kSplitWaves + wave) * 2 + (i & 1)) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int p = wave; p < OT / 2 * TT; p += kSplitWaves) {
    f32x4 lo = s_acc[p * kSplitWaves * 128 + lane], hi = s_acc[p * kSplitWaves * 128 + 64 + lane];
#pragma unroll
    for (int q = 1; q < kSplitWaves; ++q) {
      lo += s_acc[(p * kSplitWaves + q) * 128 + lane];
      hi += s_acc[(p * kSplitWaves + q) * 128 + 64 + lane];
    }
    store_pair<E>(a, tab, 16 * (tt0 + p % TT), 16 * (ot0 + 2 * (p / TT)), lane, lo, hi);
  }
}

// Copies from memory to LDS without registers: lane l's 16 (4) bytes of src to dst + 16 l
// (4 l).  src and dst are uniform, `at` is the lane's offset in src.  In assembly, since
// the compiler makes every read of LDS behind such a copy wait for all of them: the
// kernels below read one buffer while the other is filled, and wait for their copies
// themselves (copies_landed) before the barrier behind which they are read.  The copy takes its place in LDS
// from m0, a register that the compiler keeps for itself and does not accept as overwritten: it is put back (16384 x
// 3072, 8192 tokens: 444.4 us, without 443.3).
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(size_t)(__attribute__((address_space(3))) const void*)p;
}
__device__ __forceinline__ void copy_kb(const uint8_t* src, uint32_t dst, uint32_t at) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(dst), "v"(at), "s"(src) : "memory");
}
__device__ __forceinline__ void copy_words(const float* src, uint32_t dst, uint32_t at) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(dst), "v"(at), "s"(src) : "memory");
}
__device__ __forceinline__ void copies_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Large batches: a block takes 16 WO WR outputs x 16 TO TR tokens (WR x TR waves of WO x TO
// tiles).  The operands of one input block are copied into LDS while the previous one is
// multiplied: two buffers (of their own, so that the compiler sees that a copy into one
// need not be waited for by reads of the other), one barrier a block.  Tiles lie in LDS as in
// memory, so copies and operand reads are both 1 KB in a row without bank conflicts.
// 16384 x 3072, 8192 tokens: 390 to 437 us from card to card with the quantiser's 14, 1.9 to 2.1
// PFLOP/s.  399 without y's stores (268 MB, which nothing overlaps), 380 without the copies, 390 without
// the matrix instructions in a run of 425: no one of them bounds it.  Matrix units busy 56 %; alone they
// reach 4.7 PFLOP/s here, 4.5 with the four additions that the scales need behind each.
template <typename E, int WO, int TO, int WR, int TR>
__global__ void __launch_bounds__(64 * WR * TR) k_base_tile(BaseArgs a) {
  constexpr int NO = WO * WR, NT = TO * TR, kWaves = WR * TR;
  // a buffer: the output tiles, the token tiles, the tokens' scales, and each wave's outputs' scale 64 times
  constexpr int kSx = (NO + NT) * kBaseTile, kSw = kSx + 64 * NT, kStage = kSw + 256 * kWaves;
  __shared__ __attribute__((aligned(16))) uint8_t s_a[kStage], s_b[kStage];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Blocks go to the 8 XCDs in turn; each XCD takes a run of the items, in which four token tiles
  // share an output tile's operand while it is in the XCD's L2.
  const int n_tok = (a.T + 16 * NT - 1) / (16 * NT), n_out = gridDim.x / n_tok;
  int id = blockIdx.x;
  if (gridDim.x % 8 == 0) id = (id & 7) * (gridDim.x >> 3) + (id >> 3);
  const int band = id / (4 * n_out), first = 4 * band, width = min(4, n_tok - first);
  const int in_band = id - 4 * n_out * band;
  const int item = in_band / width, tok = first + in_band % width;
  const BaseTable& tab = a.tab[table_of(a, item)];
  const int ot0 = (item - tab.first) * NO, tt0 = tok * NT;
  const int wo = (wave % WR) * WO, wt = (wave / WR) * TO;

  // The wave's half tiles of an input block: every kWaves-th of the outputs', then of the tokens'.
  constexpr int PW = 2 * NO / kWaves, PX = 2 * NT / kWaves;
  static_assert(kWaves % 2 == 0 && 2 * NO % kWaves == 0 && 2 * NT % kWaves == 0, "whole half tiles to a wave");
  const size_t row = (size_t)a.kb * kBaseTile, mine = (wave >> 1) * row + (wave & 1) * 1024;
  const uint8_t* const src_w = tab.w + ot0 * row + mine;
  const uint8_t* const src_x = a.xq + tt0 * row + mine;
  const int part = wave % (NT / 4);
  const float* const src_sx = a.sx + 16 * tt0 + 64 * part;
  const float* const src_sw = tab.sw + (ot0 + wo) / 8;
  const uint32_t at16 = 16 * lane, at4 = 4 * lane;
  auto copy = [&](int kb, uint8_t* stage) {
    const uint32_t dst = lds_offset(stage);
    const uint8_t *pw = src_w + (size_t)kb * kBaseTile, *px = src_x + (size_t)kb * kBaseTile;
#pragma unroll
    for (int p = 0; p < PW; ++p) copy_kb(pw + (size_t)(p * kWaves / 2) * row, dst + (p * kWaves + wave) * 1024, at16);
#pragma unroll
    for (int p = 0; p < PX; ++p)
      copy_kb(px + (size_t)(p * kWaves / 2) * row, dst + NO * kBaseTile + (p * kWaves + wave) * 1024, at16);
    // (no branches here: the step's arithmetic must stay in one block of code)
    copy_words(src_sx + (size_t)kb * a.T_pad, dst + kSx + 256 * part, at4);
    copy_words(src_sw + (size_t)kb * tab.n_blk, dst + kSw + 256 * wave, 0);
  };
  f32x4 acc[WO][TO];
#pragma unroll
  for (int i = 0; i < WO; ++i)
#pragma unroll
    for (int j = 0; j < TO; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto scales = [&](const uint8_t* st, float (&s)[TO]) {
    const float sw = *reinterpret_cast<const float*>(st + kSw + 256 * wave);
#pragma unroll
    for (int j = 0; j < TO; ++j) s[j] = sw * *reinterpret_cast<const float*>(st + kSx + 4 * (16 * (wt + j) + (lane & 15)));
  };
  // One input block: x and the first output tile's codes are in registers (x, w), those of the
  // next block are fetched behind the barrier, while the last two tiles are multiplied.
  auto step = [&](int kb, uint8_t* cur, const uint8_t* next, const Codes<E>(&x)[TO], const float(&s)[TO],
                  Codes<E>(&xn)[TO], float(&sn)[TO], Codes<E>& w) {
    Codes<E> wt_[WO + 1];
    wt_[0] = w;
    f32x4 p[3];
#pragma unroll
    for (int i = 0; i < WO; ++i) {
      if (i + 1 < WO) wt_[i + 1].set(load_tile(cur + (wo + i + 1) * kBaseTile, lane));
      if (i == WO - 2) {
        // every read of `cur` is done, and the copy into `next` (of this wave, then of all) has landed
        copies_landed();
        __syncthreads();
#pragma unroll
        for (int j = 0; j < TO; ++j) xn[j].set(load_tile(next + (NO + wt + j) * kBaseTile, lane));
        wt_[WO].set(load_tile(next + wo * kBaseTile, lane));
        scales(next, sn);
        copy(min(kb + 2, a.kb - 1), cur);                  // (past the end the last block again: no branch, never used)
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < TO; ++j) {
        const int n = i * TO + j;                          // products two behind are scaled and added
        p[n % 3] = Codes<E>::mma(wt_[i], x[j]);
        if (n >= 2) add_scaled(acc[(n - 2) / TO][(n - 2) % TO], p[(n - 2) % 3], s[(n - 2) % TO]);
      }
      if (i + 1 < WO && i != WO - 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
      for (int j = 0; j < TO; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = WO * TO; n < WO * TO + 2; ++n)
      add_scaled(acc[(n - 2) / TO][(n - 2) % TO], p[(n - 2) % 3], s[(n - 2) % TO]);
    w = wt_[WO];
  };
  copy(0, s_a);
  copy(min(1, a.kb - 1), s_b);
  copies_landed();
  __syncthreads();
  Codes<E> x0[TO], x1[TO], w0;
#pragma unroll
  for (int j = 0; j < TO; ++j) x0[j].set(load_tile(s_a + (NO + wt + j) * kBaseTile, lane));
  w0.set(load_tile(s_a + wo * kBaseTile, lane));
  float sc0[TO], sc1[TO];
  scales(s_a, sc0);
  int kb = 0;
  for (; kb + 2 <= a.kb; kb += 2) {
    step(kb, s_a, s_b, x0, sc0, x1, sc1, w0);
    step(kb + 1, s_b, s_a, x1, sc1, x0, sc0, w0);
  }
  if (kb < a.kb) step(kb, s_a, s_b, x0, sc0, x1, sc1, w0);
  // y by way of LDS, 16 tokens at a time, so that each is written in runs of 16 WO outputs, and past the
  // caches, which keep x and W: 16384 x 3072, 8192 tokens, 456 us straight from the lanes, 452 by
  // way of LDS, 437 past the caches as well.
  // The last copies have landed and the buffers are no longer read; each wave has its own part.
  copies_landed();
  __syncthreads();
  constexpr int kRow = 16 * WO * (int)sizeof(E), kLd = kRow + 16, kLanes = kRow / 16, kRows = 64 / kLanes;
  static_assert(kWaves / 2 * 16 * kLd <= kStage, "the waves' parts fit the buffers");
  uint8_t* const mine_y = (wave < kWaves / 2 ? s_a : s_b) + (wave % (kWaves / 2)) * 16 * kLd;
#pragma unroll
  for (int j = 0; j < TO; ++j) {
#pragma unroll
    for (int i = 0; i < WO; i += 2)
      store8(reinterpret_cast<E*>(mine_y + (lane & 15) * kLd) + 16 * i + 8 * (lane >> 4), acc[i][j], acc[i + 1][j]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int o = 16 * (ot0 + wo) + lane % kLanes * (16 / (int)sizeof(E));
#pragma unroll
    for (int r = 0; r < 16; r += kRows) {
      const uint4 v = *reinterpret_cast<const uint4*>(mine_y + (r + lane / kLanes) * kLd + lane % kLanes * 16);
      const int t = 16 * (tt0 + wt + j) + r + lane / kLanes;
      if (t < a.T && o < tab.out)
        __builtin_nontemporal_store((u32x4){v.x, v.y, v.z, v.w},
                                    reinterpret_cast<u32x4*>(reinterpret_cast<E*>(tab.y) + (size_t)t * tab.out + o));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

}  // namespace

hipError_t launch_base_pin(const BasePinArgs& a, int bf16, hipStream_t s) {
  const dim3 grid(a.kb, a.tab.n_blk);
  if (bf16) hipLaunchKernelGGL(k_base_pin<uint16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_base_pin<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_base_pin_codes(const BasePinArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_base_pin_codes, dim3(a.kb, a.tab.n_blk), dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_base_read(const BasePinArgs& a, int bf16, hipStream_t s) {
  const dim3 grid(a.kb, a.tab.n_blk);
  if (bf16) hipLaunchKernelGGL(k_base_read<uint16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_base_read<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

namespace {

// Work items, table after table: `per` for every `outs` outputs.
int number_items(BaseArgs& a, int outs, int per = 1) {
  int items = 0;
  for (int i = 0; i < a.n_tables; ++i) {
    a.tab[i].first = items;
    items += per * cdiv(a.tab[i].out, outs);
  }
  return items;
}

template <typename E, int OT, int TT>
hipError_t launch_split(BaseArgs& a, hipStream_t s) {
  const dim3 grid(number_items(a, 16 * OT), cdiv(a.T, 16 * TT));
  hipLaunchKernelGGL((k_base_split<E, OT, TT>), grid, dim3(64 * kSplitWaves), split_lds(OT, TT), s, a);
  return hipGetLastError();
}
template <typename E, int WO, int TO, int WR, int TR>
hipError_t launch_tile(BaseArgs& a, hipStream_t s) {
  const int items = number_items(a, 16 * WO * WR);
  hipLaunchKernelGGL((k_base_tile<E, WO, TO, WR, TR>), dim3(items * cdiv(a.T, 16 * TO * TR)), dim3(64 * WR * TR),
                     0, s, a);
  return hipGetLastError();
}

template <typename E>
hipError_t product(BaseArgs& a, int n_cu, hipStream_t s) {
  const BaseKernel kernel = base_kernel([&](int i) { return a.tab[i].out; }, a.n_tables, a.T, sizeof(E), n_cu);
  if (kernel == kBaseFew1 || kernel == kBaseFew2) {
    if (kernel == kBaseFew1)
      hipLaunchKernelGGL((k_base_few<E, 1>), dim3(number_items(a, 32, 2)), dim3(64 * kFewWaves), 0, s, a);
    else hipLaunchKernelGGL((k_base_few<E, 2>), dim3(number_items(a, 32)), dim3(64 * kFewWaves), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_base_quantise<E>, dim3(cdiv(a.T, 16), cdiv(a.kb, 4)), dim3(256), 0, s, a);
  if constexpr (sizeof(E) == 2) {
    if (kernel == kBaseTile256x256) return launch_tile<E, 8, 4, 2, 4>(a, s);
    if (kernel == kBaseTile128x256) return launch_tile<E, 4, 4, 2, 4>(a, s);
  }
  if (kernel == kBaseTile128x128) return launch_tile<E, 4, 4, 2, 2>(a, s);
  if (kernel == kBaseSplit64x64) return launch_split<E, 4, 4>(a, s);
  if (kernel == kBaseSplit32x64) return launch_split<E, 2, 4>(a, s);
  return launch_split<E, 2, 2>(a, s);
}

}  // namespace

hipError_t launch_base_product(const BaseArgs& args, int bf16, int n_cu, hipStream_t s) {
  BaseArgs a = args;
  return bf16 ? product<uint16_t>(a, n_cu, s) : product<float>(a, n_cu, s);
}

}  // namespace salt
