// Host-side check of the dense path's index arithmetic (no GPU call is made).
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../paper_2602_01801_b200/csrc/dense.h"

using namespace fastar;

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

int main() {
  // the end of the keys that a position sees
  for (int len = 1; len < 70; ++len)
    for (int f = 0; f < 75; ++f)
      for (int pos = 0; pos < len; ++pos) {
        int end = 0;
        for (int j = 0; j < len; ++j)
          if (f == 0 || j / f <= pos / f) end = j + 1;
        CHECK(visible_end(pos, len, f) == end);
      }
  CHECK(visible_end(INT32_MAX - 1, INT32_MAX, INT32_MAX) == INT32_MAX);
  CHECK(visible_end(INT32_MAX - 1, INT32_MAX, 1) == INT32_MAX);
  CHECK(visible_end(INT32_MAX - 2, INT32_MAX, 2) == INT32_MAX - 1 || visible_end(INT32_MAX - 2, INT32_MAX, 2) == INT32_MAX);
  CHECK(pages_of(INT32_MAX, 64) == (1 << 25) && pages_of(0, 64) == 0 && pages_of(1, 64) == 1 && pages_of(64, 64) == 1 && pages_of(65, 64) == 2);
  // sequences
  DenseSeq s;
  CHECK(check_seq(s, 0, 5, 9, 10, 5, 9) == 1 && s.t0 == 0 && s.n == 5 && s.len == 9);
  CHECK(check_seq(s, 3, 3, 9, 10, 5, 9) == 0 && s.n == 0);
  CHECK(check_seq(s, 3, 5, -1, 10, 5, 9) == 0 && s.n == 0);
  CHECK(check_seq(s, 3, 5, 10, 10, 5, 9) == -1 && s.n == 0);
  CHECK(check_seq(s, 3, 9, 9, 10, 5, 9) == -1);
  CHECK(check_seq(s, 3, 5, 1, 10, 5, 9) == -1);
  CHECK(check_seq(s, 5, 3, 9, 10, 5, 9) == -1);
  CHECK(check_seq(s, -1, 3, 9, 10, 5, 9) == -1);
  CHECK(check_seq(s, 8, 11, 9, 10, 5, 9) == -1);
  CHECK(check_seq(s, INT32_MIN, INT32_MAX, 9, INT32_MAX, 5, 9) == -1);
  // scales: the least power of two that fits
  for (int e = -149; e <= 127; ++e)
    for (int m = 0; m < 64; ++m) {
      const float a = std::ldexp(1.f + m / 64.f, e);
      if (!(a > 0.f) || std::isinf(a)) continue;
      uint32_t bits;
      std::memcpy(&bits, &a, 4);
      const int x = scale_exp_of(bits);
      CHECK(x >= kMinScaleExp && x <= 120);
      CHECK(static_cast<double>(a) <= 448.0 * std::ldexp(1.0, x));
      if (x > kMinScaleExp) CHECK(static_cast<double>(a) > 448.0 * std::ldexp(1.0, x - 1));
    }
  CHECK(scale_exp_of(0) == kMinScaleExp);
  // touched pages of n tokens from `past` on: no more than n, nor than (n - 2) / page + 2
  for (int past = 0; past < 300; ++past)
    for (int n = 1; n < 300; ++n) {
      const int pages = pages_of(past + n, 64) - past / 64;
      CHECK(pages <= n && pages <= (n + 126) / 64 && pages * 64 <= n + 126);
    }
  std::printf("ok\n");
  return 0;
}
