// Host build of the search for a token's document (xhc_spans.h).
//
// Input, one case per line: n (documents) t m, then m pairs i s: from index i on
// the starts are s (0 in front of the first pair); the last index is n.  The
// starts are in memory that is only touched where it is written or read, so n may
// be as large as its type.  Output, one line per case: the index that is found.
#include <sys/mman.h>

#include <cstdio>

#include "xhc_spans.h"

int main() {
  long n;
  int t, m;
  while (std::scanf("%ld %d %d", &n, &t, &m) == 3) {
    const size_t bytes = ((size_t)n + 1) * 4;
    int32_t* starts = static_cast<int32_t*>(
        mmap(nullptr, bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
    if (starts == MAP_FAILED) return 2;
    long from[64];
    int value[64];
    for (int k = 0; k < m; ++k)
      if (std::scanf("%ld %d", &from[k], &value[k]) != 2 || m > 64) return 2;
    for (int k = 0; k < m; ++k)
      for (long i = from[k]; i < (k + 1 < m ? from[k + 1] : n + 1); ++i) starts[i] = value[k];
    std::printf("%d\n", xhc::last_start(starts, (int)n, t));
    munmap(starts, bytes);
  }
  return 0;
}
