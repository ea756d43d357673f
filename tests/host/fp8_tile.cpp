// The 8-bit product's launcher on the host: reads "M N K wide" by the line, writes the width of the tiles it takes (`wide`: 32-bit
// results).  Built by tests/test_fp8_choice.py.
#include "../../paper_2110_13005_amd/csrc/host_logic.h"

#include <cstdio>

int main() {
  long long M, N, K;
  int wide;
  while (std::scanf("%lld %lld %lld %d", &M, &N, &K, &wide) == 4)
    std::printf("%d\n", 64 << axonn::host::choose_fp8_tile(M, N, (K + 127) / 128, wide != 0));
  return 0;
}
