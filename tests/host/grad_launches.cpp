// Host build of the launches of a gradient norm or clip (xhc_grad_launches.h),
// recorded instead of made.
//
// Input, one case per line: clip (0 or 1), the number of tensors, then each
// one's elements.  Tensor i lies at address i + 1, its output at i + 1 + 2^20.
// Output, per case: "places P chunk E", then a line per launch: "squares
// part_at grid" and "scale grid own chunks", each followed by "i elements
// first" of its tensors, and "norm chunks clip"; a last line "end status".
#include <cstdio>
#include <vector>

#include "xhc_grad_launches.h"

struct Record {
  static void tensors(const xhc::GradBatch& b) {
    for (int i = 0; i < b.n; ++i) {
      const long long at = (long long)b.src[i] - 1;
      std::printf(" %lld %lld %d", b.dst[i] == 0 || b.dst[i] == b.src[i] + (1 << 20) ? at : -1, (long long)b.count[i],
                  b.first[i]);
    }
    std::printf("\n");
  }
  hipError_t squares(const xhc::GradBatch& b) {
    std::printf("squares %lld %d", (long long)b.part_at, b.first[b.n]);
    tensors(b);
    return hipSuccess;
  }
  hipError_t norm(int64_t chunks, bool clip) {
    std::printf("norm %lld %d\n", (long long)chunks, (int)clip);
    return hipSuccess;
  }
  hipError_t scale(const xhc::GradBatch& b, bool own, int64_t chunks) {
    std::printf("scale %d %d %lld", b.first[b.n], (int)own, (long long)chunks);
    tensors(b);
    return hipSuccess;
  }
};

int main() {
  int clip, n;
  while (std::scanf("%d %d", &clip, &n) == 2) {
    std::vector<const void*> grads(n);
    std::vector<void*> outs(n);
    std::vector<int64_t> counts(n);
    std::vector<int32_t> dtypes(n, XHC_F32);
    for (int i = 0; i < n; ++i) {
      long long c;
      if (std::scanf("%lld", &c) != 1) return 1;
      counts[i] = c;
      grads[i] = reinterpret_cast<const void*>((uintptr_t)i + 1);
      outs[i] = reinterpret_cast<void*>((uintptr_t)i + 1 + (1 << 20));
    }
    std::printf("places %zu chunk %lld\n", xhc::grad_places(n), (long long)xhc::chunk_elems(n, counts.data()));
    Record r;
    static void* none[1];
    const hipError_t e = xhc::grad_launches(r, n, grads.data(), counts.data(), dtypes.data(),
                                            clip ? (n ? outs.data() : none) : nullptr);
    std::printf("end %d\n", (int)e);
  }
  return 0;
}
