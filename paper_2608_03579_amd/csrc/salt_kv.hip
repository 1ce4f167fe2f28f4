// The paged KV cache: k and v of a step quantised as they are written, and read back.
//
// Per token and kv head, k and v apart, over the vector's D values:
//   e4m3: s = smallest power of two with amax / s <= 448 (1 for a zero vector, at least
//         2^-100), code = e4m3(x / s).  A power of two costs an 8-bit float nothing but
//         a binade of its range, and code * s is exact in bf16.
//   int8: s = max(amax * (1/127), 2^-100), code = rint(x * (1 / s)) in [-127, 127].
// Sixteen lanes hold one vector pair (k, v): one pass over the data, the maximum by
// four lane exchanges.  Bound by memory traffic and, for a decode step, by the launch: 256 tokens of
// 8 x 128 values written in 3.3 us, 8192 in 12.4 (4.2 TB/s of k, v and codes), 70 MB of codes read back as
// 133 MB of bf16 in 32 to 44 us (4.7 to 6.3 TB/s from card to card).
#include <hip/hip_runtime.h>

#include "salt_device.h"
#include "salt_layout.h"
#include "salt_serve.h"

namespace salt {
namespace {

constexpr uint32_t kInfBits = 0x7f800000u;

// N values (N / 4 code words) of a lane; loads and stores of 4 values or more.
template <typename E, int N>
__device__ __forceinline__ void load_values(const E* p, float (&v)[N]) {
  if constexpr (sizeof(E) == 4) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const float4 w = *reinterpret_cast<const float4*>(p + j);
      v[j] = w.x; v[j + 1] = w.y; v[j + 2] = w.z; v[j + 3] = w.w;
    }
  } else if constexpr (N == 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = bf_lo(w.x); v[1] = bf_hi(w.x); v[2] = bf_lo(w.y); v[3] = bf_hi(w.y);
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 8) Ops<E>::to_f32(Ops<E>::load(p + j), v + j);
  }
}
template <typename E, int N>
__device__ __forceinline__ void store_values(E* p, const float (&v)[N]) {
  if constexpr (sizeof(E) == 4) {
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  } else if constexpr (N == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 8) Ops<E>::store(p + j, v + j);
  }
}
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&w)[N / 4]) {
  if constexpr (N == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
  else if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <int N>
__device__ __forceinline__ void load_codes(const uint8_t* p, uint32_t (&w)[N / 4]) {
  if constexpr (N == 4) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 8) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  }
}

// Codes and scale of one vector, N of its values in each of 16 lanes.  The bits of the
// magnitudes order like the magnitudes, with infinities and NaNs above every number.
template <int FMT, int N>
__device__ __forceinline__ float quantise_vec(const float (&v)[N], uint32_t (&w)[N / 4]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
  for (int m = 1; m < 16; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (top >= kInfBits) {
#pragma unroll
    for (int j = 0; j < N / 4; ++j) w[j] = 0;
    return __uint_as_float(0x7fc00000u);
  }
  if constexpr (FMT == kKvInt8) {
    const float s = fmaxf(__uint_as_float(top) * (1.0f / 127.0f), 0x1p-100f), r = 1.0f / s;
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
      w[j] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int q = min(max((int)rintf(v[4 * j + e] * r), -127), 127);
        w[j] |= ((uint32_t)q & 0xffu) << (8 * e);
      }
    }
    return s;
  } else {
    // 448 = 1.75 * 2^8
    int e2 = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e2 = top == 0 ? 0 : max(e2, -100);
    const float r = __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j] * r, v[4 * j + 1] * r, 0, false);
      w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j + 2] * r, v[4 * j + 3] * r, lo, true);
    }
    return __uint_as_float((uint32_t)(127 + e2) << 23);
  }
}
template <int FMT, int N>
__device__ __forceinline__ void read_vec(const uint32_t (&w)[N / 4], float s, float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    if constexpr (FMT == kKvInt8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = (float)((int)(w[j] << (24 - 8 * e)) >> 24) * s;
    } else {
      v[4 * j] = __builtin_amdgcn_cvt_f32_fp8((int)w[j], 0) * s;
      v[4 * j + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[j], 1) * s;
      v[4 * j + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[j], 2) * s;
      v[4 * j + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[j], 3) * s;
    }
  }
}

// Vector of kv head h at token place `off` of page `page`, in units of vectors.
__device__ __forceinline__ size_t vec_of(const KvLayer& kv, int page, int h, int off) {
  return (((size_t)page * kv.kv_heads + h) << kv.log2_page) + off;
}

template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256) k_kv_write(KvWriteArgs a) {
  constexpr int N = D / 16;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int l = threadIdx.x & 15;
  const int t = (int)(i / a.kv.kv_heads), h = (int)(i - (int64_t)t * a.kv.kv_heads);
  if (t >= a.T) return;
  const int slot = a.slot[t];
  if (slot < 0) return;                       // (whole groups of 16 lanes leave together)
  float k[N], v[N];
  load_values<E, N>(reinterpret_cast<const E*>(a.k) + t * a.ldk + h * D + l * N, k);
  load_values<E, N>(reinterpret_cast<const E*>(a.v) + t * a.ldv + h * D + l * N, v);
  uint32_t kw[N / 4], vw[N / 4];
  float ks = quantise_vec<FMT, N>(k, kw);
  const float vs = quantise_vec<FMT, N>(v, vw);
  if (vs != vs) ks = vs;
  const size_t at = vec_of(a.kv, slot >> a.kv.log2_page, h, slot & ((1 << a.kv.log2_page) - 1));
  store_codes<N>(a.kv.k + at * D + l * N, kw);
  store_codes<N>(a.kv.v + at * D + l * N, vw);
  if (l == 0) {
    a.kv.ks[at] = ks;
    a.kv.vs[at] = vs;
  }
}

template <typename E, int D, int FMT>
__device__ __forceinline__ void read_one(const KvReadArgs& a, size_t at, int64_t row, int h, int l) {
  constexpr int N = D / 16;
  uint32_t kw[N / 4], vw[N / 4];
  load_codes<N>(a.kv.k + at * D + l * N, kw);
  load_codes<N>(a.kv.v + at * D + l * N, vw);
  const float ks = a.kv.ks[at], vs = a.kv.vs[at];
  float k[N], v[N];
  read_vec<FMT, N>(kw, ks, k);
  read_vec<FMT, N>(vw, vs, v);
  store_values<E, N>(reinterpret_cast<E*>(a.k) + row * a.ldk + h * D + l * N, k);
  store_values<E, N>(reinterpret_cast<E*>(a.v) + row * a.ldv + h * D + l * N, v);
}

// The step's tokens, in the order of q.
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256) k_kv_read_new(KvReadArgs a) {
  constexpr int N = D / 16;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int l = threadIdx.x & 15;
  const int t = (int)(i / a.kv.kv_heads), h = (int)(i - (int64_t)t * a.kv.kv_heads);
  if (t >= a.n) return;
  const int slot = a.slot[t];
  if (slot < 0) {
    const float z[N] = {};
    store_values<E, N>(reinterpret_cast<E*>(a.k) + t * a.ldk + h * D + l * N, z);
    store_values<E, N>(reinterpret_cast<E*>(a.v) + t * a.ldv + h * D + l * N, z);
    return;
  }
  read_one<E, D, FMT>(a, vec_of(a.kv, slot >> a.kv.log2_page, h, slot & ((1 << a.kv.log2_page) - 1)), t, h, l);
}

// Every own token of the sequences, page after page: a block takes 64 vector pairs of one
// page reference, which stand together in memory.
constexpr int kReadVecs = 64;
template <typename E, int D, int FMT>
__global__ void __launch_bounds__(256) k_kv_read_own(KvReadArgs a) {
  const int ref = blockIdx.x, l = threadIdx.x & 15, pt = 1 << a.kv.log2_page;
  const int page = a.page[ref], row = a.row[ref], count = a.count[ref];
#pragma unroll
  for (int q = 0; q < kReadVecs / 16; ++q) {
    const int i = blockIdx.y * kReadVecs + q * 16 + (threadIdx.x >> 4);
    const int h = i >> a.kv.log2_page, off = i & (pt - 1);
    if (h < a.kv.kv_heads && off < count) read_one<E, D, FMT>(a, vec_of(a.kv, page, h, off), row + off, h, l);
  }
}

template <typename F>
hipError_t by_type(int bf16, int dim, int format, F f) {
  auto fmt = [&](auto e, auto d) {
    if (format == kKvInt8) f(e, d, std::integral_constant<int, kKvInt8>());
    else f(e, d, std::integral_constant<int, kKvE4m3>());
  };
  auto dims = [&](auto e) {
    if (dim == 64) fmt(e, std::integral_constant<int, 64>());
    else if (dim == 128) fmt(e, std::integral_constant<int, 128>());
    else fmt(e, std::integral_constant<int, 256>());
  };
  if (bf16) dims(uint16_t());
  else dims(float());
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a, int bf16, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.T * a.kv.kv_heads + 15) / 16));
  return by_type(bf16, a.kv.dim, a.kv.format, [&](auto e, auto d, auto f) {
    hipLaunchKernelGGL((k_kv_write<decltype(e), decltype(d)::value, decltype(f)::value>), grid, dim3(256), 0, s, a);
  });
}

hipError_t launch_kv_read(const KvReadArgs& a, int bf16, hipStream_t s) {
  if (a.slot) {
    const dim3 grid((unsigned)(((int64_t)a.n * a.kv.kv_heads + 15) / 16));
    return by_type(bf16, a.kv.dim, a.kv.format, [&](auto e, auto d, auto f) {
      hipLaunchKernelGGL((k_kv_read_new<decltype(e), decltype(d)::value, decltype(f)::value>), grid, dim3(256), 0, s,
                         a);
    });
  }
  const dim3 grid(a.n, cdiv(a.kv.kv_heads << a.kv.log2_page, kReadVecs));
  return by_type(bf16, a.kv.dim, a.kv.format, [&](auto e, auto d, auto f) {
    hipLaunchKernelGGL((k_kv_read_own<decltype(e), decltype(d)::value, decltype(f)::value>), grid, dim3(256), 0, s, a);
  });
}

}  // namespace salt
