// Prints which kernel a base product takes on a device of 256 compute units (salt_base_rule.h built without HIP).
// Arguments: bytes of the type, tokens, outputs of each table.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "salt_base_rule.h"

int main(int argc, char** argv) {
  if (argc < 4) return 2;
  const char* names[] = {"few 1", "few 2", "tile 256x256", "tile 128x256", "tile 128x128", "split 64x64", "split 32x64", "split 32x32"};
  std::vector<int> outs;
  for (int i = 3; i < argc; ++i) outs.push_back(std::atoi(argv[i]));
  std::puts(names[salt::base_kernel([&](int i) { return outs[i]; }, (int)outs.size(), std::atoi(argv[2]), std::atoi(argv[1]), 256)]);
}
