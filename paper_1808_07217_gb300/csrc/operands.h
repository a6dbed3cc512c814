// Checks of the operands that the stand-alone operators' entry points share.
#pragma once
#include <algorithm>
#include <stdint.h>

namespace lsgd {

// `count` blocks of `bytes` from p, `stride` values of `elem` bytes from one to the next; at NULL: nothing.  (A workspace that is not
// used, of no bytes, counts by its address.)
struct Blocks {
  uintptr_t first, end;  // of all of them
  size_t bytes;
  int64_t stride;
  int count, elem;
  Blocks(const void* p, size_t n, int64_t gs = 0, int blocks = 1, int size = 4)
      : first(reinterpret_cast<uintptr_t>(p)), bytes(n), stride(gs), count(blocks), elem(size) {
    uint64_t span;  // (a stride may be any number: up to the last address then)
    if (__builtin_mul_overflow((uint64_t)(blocks - 1), (uint64_t)gs, &span) || span > UINTPTR_MAX / 8) end = UINTPTR_MAX;
    else end = first + elem * span + n;
    if (!p) end = 0;
  }
};
// Whether any two blocks of a and b share a byte.  Where both are several, their strides are the same.
inline bool blocks_meet(const Blocks& a, const Blocks& b) {
  if (a.first >= b.end || b.first >= a.end) return false;
  if (a.count == 1 && b.count == 1) return true;
  // block j of b lies d + t stride behind block i of a, t = j - i
  using wide = __int128;
  const wide d = (wide)b.first - (wide)a.first, na = a.bytes, nb = b.bytes;
  const wide stride = a.count > 1 ? a.elem * (wide)a.stride : b.elem * (wide)b.stride;
  const wide t = std::max<wide>(1 - a.count, (-nb - d >= 0 ? (-nb - d) / stride : -((nb + d + stride - 1) / stride)) + 1);
  return t <= b.count - 1 && d + t * stride < na;  // (t: the first that does not end before a's block)
}
// Whether anything written meets anything else of the call.
template <int W, int R>
bool any_overlap(const Blocks (&written)[W], const Blocks (&read)[R]) {
  for (int i = 0; i < W; ++i) {
    for (int j = i + 1; j < W; ++j)
      if (blocks_meet(written[i], written[j])) return true;
    for (int j = 0; j < R; ++j)
      if (blocks_meet(written[i], read[j])) return true;
  }
  return false;
}

inline bool misaligned(const void* p, int z) { return reinterpret_cast<uintptr_t>(p) % z != 0; }

}  // namespace lsgd
