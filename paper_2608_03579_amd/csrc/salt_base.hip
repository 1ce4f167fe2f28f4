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

#include "salt_device.h"
#include "salt_layout.h"
#include "salt_serve.h"

namespace salt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
constexpr float kE4m3Max = 448.f;

// Scale of a block whose largest magnitude is amax (a NaN in the block does not
// show in amax; it becomes a NaN code).
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
  // (0x7f is the scale 2^0 of the instruction's own scale operands.)
  static __device__ __forceinline__ f32x4 mma(const Codes& a, const Codes& b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0x7f7f7f7f, 0,
                                                            0x7f7f7f7f);
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
  __shared__ float s_max[4];
  const int kb = blockIdx.x, nb = blockIdx.y, tid = threadIdx.x;
  float amax = 0.f;
  for (int p = tid; p < kBaseBlock * (kBaseBlock / 8); p += 256) {
    const int k = p >> 4, o = (p & 15) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (kb * kBaseBlock + k < a.in && nb * kBaseBlock + o < a.tab.out)
      Ops<E>::to_f32(Ops<E>::load(reinterpret_cast<const E*>(a.w) + (size_t)(kb * kBaseBlock + k) * a.ld +
                                  nb * kBaseBlock + o), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s_v[k][o + e] = v[e];
      amax = fmaxf(amax, fabsf(v[e]));
    }
  }
  for (int m = 1; m < 64; m *= 2) amax = fmaxf(amax, __shfl_xor(amax, m));
  if ((tid & 63) == 0) s_max[tid >> 6] = amax;
  __syncthreads();
  const float s = block_scale(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])));
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

// One wave: 64 outputs x 64 tokens over all inputs, operands straight from memory.
template <typename E>
__global__ void __launch_bounds__(64) k_base_product(BaseArgs a) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const BaseTable& tab = a.tab[table_of(a, blockIdx.x)];
  const int o0 = (blockIdx.x - tab.first) * 64, t0 = blockIdx.y * 64;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = 0; kb < a.kb; ++kb) {
    Codes<E> w[4], x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i].set(load_tile(tab.w + ((size_t)(o0 / 16 + i) * a.kb + kb) * kBaseTile, lane));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j].set(load_tile(a.xq + ((size_t)(t0 / 16 + j) * a.kb + kb) * kBaseTile, lane));
    const float sw = tab.sw[(size_t)kb * tab.n_blk + o0 / kBaseBlock];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float s = sw * a.sx[(size_t)kb * a.T_pad + t0 + 16 * j + (lane & 15)];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 p = Codes<E>::mma(w[i], x[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], s, acc[i][j][e]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = t0 + 16 * j + (lane & 15);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int o = o0 + 16 * i + 8 * g;
      if (t < a.T && o < tab.out) store8(reinterpret_cast<E*>(tab.y) + (size_t)t * tab.out + o, acc[i][j], acc[i + 1][j]);
    }
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

hipError_t launch_base_product(const BaseArgs& args, int bf16, int n_cu, hipStream_t s) {
  (void)n_cu;
  BaseArgs a = args;
  const dim3 qgrid(cdiv(a.T, 16), cdiv(a.kb, 4));
  if (bf16) hipLaunchKernelGGL(k_base_quantise<uint16_t>, qgrid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_base_quantise<float>, qgrid, dim3(256), 0, s, a);
  int items = 0;
  for (int i = 0; i < a.n_tables; ++i) {
    a.tab[i].first = items;
    items += cdiv(a.tab[i].out, 64);
  }
  const dim3 grid(items, cdiv(a.T, 64));
  if (bf16) hipLaunchKernelGGL(k_base_product<uint16_t>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(k_base_product<float>, grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace salt
