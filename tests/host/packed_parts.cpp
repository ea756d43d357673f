// The backward pass of attention over packed sequences, as its launcher chooses it on the host: reads "T n_seq heads kv columns" by the
// line, writes the parts that share a tile of keys and whether dQ and dK / dV are one launch.  Built by tests/test_packed_parts.py.
#include "../../paper_2110_13005_amd/csrc/host_logic.h"

#include <cstdio>

int main() {
  long long T, n;
  int heads, kv, columns;
  while (std::scanf("%lld %lld %d %d %d", &T, &n, &heads, &kv, &columns) == 5)
    std::printf("%d %d\n", axonn::host::packed_parts(T, n, heads, kv, columns), axonn::host::packed_one_launch((T / 128 + n) * heads, columns));
  return 0;
}
