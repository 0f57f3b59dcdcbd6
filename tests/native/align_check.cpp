// The threads of a copy of unaligned operands, on the host: each piece is taken once, and
// threads past the last piece take none.
#include <cstdio>
#include <set>
#include <tuple>

#include "gts_linear_kernel.h"

using gts::nn::AlignArgs;
using gts::nn::align_piece;

static int check(int64_t rows_a, int64_t rows_b) {
  constexpr int E = 8;
  char memory;
  const AlignArgs none = {nullptr, 0, 0, 0, nullptr, 0};
  const AlignArgs a = rows_a ? AlignArgs{&memory, 13, rows_a, 13, &memory, 16} : none;
  const AlignArgs b = rows_b ? AlignArgs{&memory, 21, rows_b, 20, &memory, 24} : none;
  const int64_t pieces_a = rows_a * 2, pieces = pieces_a + rows_b * 3;
  std::set<std::tuple<bool, int64_t, int64_t>> seen;
  for (int64_t i = 0; i < (pieces + 255) / 256 * 256; ++i) {
    const auto p = align_piece<E>(a, b, pieces_a, i);
    if (p.there != (i < pieces)) return printf("thread %lld of %lld\n", (long long)i, (long long)pieces);
    if (!p.there) continue;
    if (p.row >= (p.second ? rows_b : rows_a) || p.col >= (p.second ? 24 : 16) || p.col % E != 0)
      return printf("thread %lld: row %lld, column %lld\n", (long long)i, (long long)p.row, (long long)p.col);
    if (!seen.insert({p.second, p.row, p.col}).second) return printf("thread %lld: taken before\n", (long long)i);
  }
  return (int64_t)seen.size() == pieces ? 0 : printf("%zu pieces of %lld\n", seen.size(), (long long)pieces);
}

int main() {
  for (int64_t a : {0, 1, 128, 300})
    for (int64_t b : {0, 1, 77, 256})
      if (check(a, b)) return 1;
  return 0;
}
