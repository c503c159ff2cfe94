// Which rows of dY the weight gradient of 8-bit activations reads without looking at their ends
// (csrc/tokens.h), walked on the CPU: every load of every such row stays inside the mini-batch's own rows,
// whose last one ends with its last column, and no more rows than need be are looked at.  The rule
// that lets a mini-batch's loads run into the next one must be reported.
#include <cstdio>
#include <initializer_list>

#include "tokens.h"

using namespace nbsgd;

constexpr int kStage = 64;  // tokens

template <typename Sure>
static bool walk(int T, int cols, int64_t ldy, int width, Sure sure) {
  const int64_t end = (int64_t)(T - 1) * ldy + cols;
  for (int c0 = 0; c0 < cols; c0 += width) {
    const int plain = sure(c0) > 0 ? sure(c0) / kStage * kStage : 0;
    for (int t = 0; t < plain; ++t)
      for (int q = 0; q < width / 8; ++q) {
        const int64_t at = t * ldy + c0 + (8 * q < cols - c0 ? 8 * q : 0);
        if (at < 0 || at + 8 > end) return false;
      }
  }
  return true;
}

int main() {
  bool reported = false;
  for (int T = 1; T <= 200; T += T < 60 ? 13 : 1)
    for (int cols = 1; cols <= 300; cols += cols < 40 ? 1 : 29)
      for (int64_t gap : {0, 1, 3, 8, 200})
        for (int width : {128, 256}) {
          const int border = act8_border(T, cols + gap);
          auto sure = [&](int c0) { return act8_sure(T, border, c0, width, cols); };
          if (!walk(T, cols, cols + gap, width, sure)) {
            std::printf("T=%d cols=%d gap=%d width=%d: read behind the mini-batch\n", T, cols, (int)gap, width);
            return 1;
          }
          for (int c0 = 0; c0 < cols; c0 += width)
            if (sure(c0) < T - 7 || (cols % 8 == 0 && sure(c0) != T) || (cols + gap >= 7 && sure(c0) < T - 1)) {
              std::printf("T=%d cols=%d gap=%d: only %d rows\n", T, cols, (int)gap, sure(c0));
              return 1;
            }
          reported |= !walk(T, cols, cols + gap, width, [&](int) { return T; });
        }
  if (!reported) return std::printf("the planted mistake was not reported\n"), 1;
  std::printf("ok\n");
  return 0;
}
