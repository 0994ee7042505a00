// The host side of the gradient norm and clip: chunks, tables and the order of
// launches (also run by a CPU test, which records the launches).
#pragma once

#include "xhc.h"
#include "xhc_launch.h"

namespace xhc {

constexpr int64_t kChunks = 16384;

// Tensors of one launch.  first[i]: the launch's first chunk of tensor i;
// first[n]: its chunks.  28 bytes a tensor, under the 4 KiB of a launch's arguments.
struct GradBatch {
  uint64_t src[kGradBatch], dst[kGradBatch];
  int64_t count[kGradBatch];
  int32_t first[kGradBatch + 1];
  uint64_t f32[kGradBatch / 64];   // a bit for each tensor: fp32, else bf16
  int32_t n;
  int32_t chunk;                   // elements, a multiple of 8
  int64_t part_at;                 // the launch's first chunk among all
};
static_assert(sizeof(GradBatch) + 64 <= 4096, "the arguments of a launch");

// Elements per chunk: about kChunks chunks in all, and not under 8192 elements,
// below which a workgroup's start costs more than its bytes.  (With 4096 chunks
// the last workgroups run long alone: the clip pass over 617 MB 240 us, 210 with
// 16384; their sum then takes 7 us instead of 5.)  The total is divided rounding
// up, so that there are kChunks whole chunks at most.
inline int64_t chunk_elems(int n, const int64_t* counts) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += counts[i];
  int64_t c = ((total + kChunks - 1) / kChunks + 2047) / 2048 * 2048;
  return c < 8192 ? 8192 : c;
}

// the table of the tensors from i on, as many as it takes; the tensor after them
inline int fill_batch(GradBatch& b, int i, int n, const void* const* grads, void* const* outs, const int64_t* counts,
                      const int32_t* dtypes, int64_t chunk, int64_t part_at) {
  b.n = 0;
  b.chunk = (int32_t)chunk;
  b.part_at = part_at;
  for (int w = 0; w < kGradBatch / 64; ++w) b.f32[w] = 0;
  b.first[0] = 0;
  for (; i < n && b.n < kGradBatch; ++i) {
    if (counts[i] == 0) continue;
    b.src[b.n] = (uint64_t)(uintptr_t)grads[i];
    b.dst[b.n] = outs ? (uint64_t)(uintptr_t)outs[i] : 0;
    b.count[b.n] = counts[i];
    if (dtypes[i] == XHC_F32) b.f32[b.n / 64] |= 1ull << (b.n % 64);
    b.first[b.n + 1] = b.first[b.n] + (int32_t)((counts[i] + chunk - 1) / chunk);
    ++b.n;
  }
  return i;
}

// the factor, then the chunks' sums: at most kChunks whole chunks and a last one for each tensor
inline size_t grad_places(int n) { return (size_t)kChunks + n; }

// Few chunks: every workgroup of the clip adds them itself, in the same order,
// instead of waiting for a launch that does (ten small tensors 8.9 us of kernels,
// 10 in three launches, and the time between two).
constexpr int kOwnSum = 512;

// The launches of a norm (outs null) or a clip, through
//   L::squares(table)                 the chunks' sums
//   L::norm(chunks, clip)             their sum, and the factor of a clip
//   L::scale(table, own, chunks)      own: the sums are still to be added
template <class L>
hipError_t grad_launches(L& launch, int n, const void* const* grads, const int64_t* counts, const int32_t* dtypes,
                         void* const* outs) {
  const int64_t chunk = chunk_elems(n, counts);
  // empty tensors behind the last other one would make a table of their own, with no chunk
  while (n > 0 && counts[n - 1] == 0) --n;
  GradBatch b;
  int64_t chunks = 0;
  int starts[kMaxGrads / kGradBatch + 1], batches = 0;   // the first tensor of each launch
  for (int i = 0; i < n;) {
    const int at = i;
    i = fill_batch(b, i, n, grads, outs, counts, dtypes, chunk, chunks);
    starts[batches++] = at;
    if (hipError_t e = launch.squares(b); e != hipSuccess) return e;
    chunks += b.first[b.n];
  }
  const bool own = outs && batches == 1 && chunks <= kOwnSum;
  if (!own)
    if (hipError_t e = launch.norm(chunks, outs != nullptr); e != hipSuccess || !outs) return e;
  // the last launch's tensors first; its table is still there
  for (int k = batches - 1; k >= 0; --k) {
    if (k < batches - 1) fill_batch(b, starts[k], n, grads, outs, counts, dtypes, chunk, 0);
    if (hipError_t e = launch.scale(b, own, chunks); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace xhc
