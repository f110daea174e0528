// Whether decode attention over the 8-bit cache deals its workgroups out by sequence length. Lines of "B H D block_size max_blocks ranges wide" on stdin, 1 or 0 a line on stdout;
// 256 CUs, no device. Test infrastructure.
#include <stdio.h>

#include "../../include/mlt.h"
#include "../../paper_2503_14985_amd/csrc/mlt_internal.h"

using namespace mlt;

int main() {
  long long B, H, D, block, blocks, ranges;
  int wide;
  while (scanf("%lld %lld %lld %lld %lld %lld %d", &B, &H, &D, &block, &blocks, &ranges, &wide) == 7) {
    PagedFp8Args a{};
    a.B = B; a.Hq = H; a.H = H; a.D = D; a.block_size = block; a.max_blocks = blocks; a.num_blocks = 1 << 20;
    printf("%d\n", paged_fp8_by_length(a, B * H * ranges, ranges, wide != 0, 256) ? 1 : 0);
  }
  return 0;
}
