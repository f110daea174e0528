// Which rows of the scales and zero points the tile kernel of mlt_gemm_w4 reads, by the expressions that the kernel has (gemm_4bit.h), on the host: for every K, group, chunk and lane, none behind
// the last row, and every row there is. Prints the number of row reads checked, or the first one that is wrong. Test infrastructure.
#include <stdio.h>

#include "../../paper_2503_14985_amd/csrc/gemm_4bit.h"

using namespace mlt;

template <int G> long long check(int K) {
  constexpr int KC = 128, NG = KC / G;
  const int rows = (K + G - 1) / G, last_group = (K - 1) / G;
  long long n = 0;
  for (int t = 0; t * KC < K; ++t) {
    const int k0 = t * KC;
    const bool tail = K - k0 < KC;
    bool seen[NG] = {};
    for (int lane = 0; lane < 64; ++lane) {
      const int g = lane >> 4;
      if (tail && !w4t_group_there<G>(k0, g, last_group)) continue;   // (a zero goes to LDS instead)
      const int row = t * NG + w4t_group<G>(g);
      if (row < 0 || row >= rows) {
        printf("K %d group %d chunk %d lane %d reads row %d of %d\n", K, G, t, lane, row, rows);
        return -1;
      }
      if (g < NG) seen[g] = row == t * NG + g;                        // what the products take: group q from lanes 16 q .. 16 q + 15
      ++n;
    }
    for (int q = 0; q < NG; ++q)
      if (t * NG + q < rows && !seen[q]) {
        printf("K %d group %d chunk %d: group %d is not read\n", K, G, t, q);
        return -1;
      }
  }
  return n;
}

int main() {
  long long n = 0;
  for (int K = 32; K <= 8192 + 96; K += 32) {
    const long long a = check<32>(K), b = check<64>(K), c = check<128>(K);
    if (a < 0 || b < 0 || c < 0) return 1;
    n += a + b + c;
  }
  printf("%lld\n", n);
  return 0;
}
