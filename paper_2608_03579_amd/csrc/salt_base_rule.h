// Which kernel a base product takes (salt_base.hip).  Host arithmetic on sizes alone: no HIP types.
#pragma once

#include <stdint.h>

namespace salt {

// kBaseFew1, kBaseFew2: k_base_few with one and two tiles of 16 outputs to a block.  The others by the
// outputs x tokens of a block: kBaseTile* walk all inputs in each block, kBaseSplit* split them over its waves.
enum BaseKernel {
  kBaseFew1, kBaseFew2, kBaseTile256x256, kBaseTile128x256, kBaseTile128x128, kBaseSplit64x64, kBaseSplit32x64,
  kBaseSplit32x32
};

// The largest tile whose blocks still fill the device, since a larger one reads less per product.  us
// of one product (quantised x included), by tile; bf16:
//   outputs x inputs, tokens    256 x 256   128 x 256   128 x 128   64 x 64   32 x 64   32 x 32
//   16384 x 3072, 1024               57          64          76       136       130       214
//   16384 x 3072,  512               48          36          41        73        69       110
//    4096 x 4096, 2048               64          49          54        71        82        95
//    4096 x 4096,  256               54          35          32        14        16        18
//    4096 x 4096,  128               51          33          31        12        11        12
//    4096 x 4096,   64               50          32          30        12        11        10
// fp32 (whose bf16 operands take twice the registers: no tiles above 128 x 128):
//   16384 x 3072, 1024                                       144       156       160       220
//   16384 x 3072,  512                                        73        82        83       114
//    4096 x 4096, 2048                                        97        92       100       107
//    4096 x 4096, 1024                                        51        49        54        55
//    4096 x 4096,  256                                        47        18        18        19
//    2576 x 2056,  203                                        28        12        12        13
//    4096 x 4096,  128                                        46        15        12        13
//    4096 x 4096,   64                                        46        15        11         9
//
// Few tokens: no launch ahead of the product's.  28672 x 4096 of one token 25 us in this way and
// 36 behind the quantiser, 3072 x 3072 4.6 and 7.5, of 16 tokens 5.8 and 7.7; in fp32, with
// twice the x to read in every block, 8 tokens 6.5 and 7.3, 16 tokens 8.7 and 7.6.  Two
// output tiles to a block where one each would not run at once (6144 x 4096: 6.0 and 8.3 us).
//
// out(i), i < n: the tables' outputs.  esize: bytes of the context's type.
template <typename Out>
inline BaseKernel base_kernel(Out out, int n, int T, int esize, int n_cu) {
  auto blocks = [&](int outs, int toks) {
    int64_t k = 0;
    for (int i = 0; i < n; ++i) k += (out(i) + outs - 1) / outs;
    return k * ((T + toks - 1) / toks);
  };
  if (T <= (esize == 2 ? 16 : 8)) return blocks(16, 16) <= n_cu ? kBaseFew1 : kBaseFew2;
  const int64_t most = (int64_t)n_cu * 7 / 10, some = (int64_t)n_cu * 6 / 10;
  if (esize == 2 && blocks(256, 256) >= most) return kBaseTile256x256;
  if (esize == 2 && blocks(128, 256) >= most) return kBaseTile128x256;
  if (blocks(128, 128) >= most) return kBaseTile128x128;
  if (blocks(64, 64) >= some) return kBaseSplit64x64;
  return blocks(32, 64) >= some ? kBaseSplit32x64 : kBaseSplit32x32;
}

}  // namespace salt
