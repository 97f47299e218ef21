// Where the kernel that writes keys takes a channel's angle from, for pairs of halves: always one of the dims / 2 that were computed for
// the token, for channels behind the turned ones too, and for a turned channel its pair's.
#include <stdio.h>

#include "lq_deal_paged.h"

using namespace lq;

#define CHECK(x)                                                                     \
  do {                                                                               \
    if (!(x)) {                                                                      \
      printf("line %d: %s (d %d, dims %d, channel %d)\n", __LINE__, #x, d, dims, c); \
      return 1;                                                                      \
    }                                                                                \
  } while (0)

int main() {
  const int ds[] = {64, 96, 128};
  for (int d : ds)
    for (int dims = 2; dims <= d; dims += 2)
      for (int c = 0; c < d; ++c) {
        const int pairs = dims / 2, at = angle_of(c, dims, 1);
        CHECK(at >= 0 && at < pairs);
        if (c < dims) CHECK(at == c % pairs);
        // halves that are whole pieces of eight channels: a piece's angles follow each other
        if (dims % 16 == 0 && c % 8 == 0) {
          const int piece = angle_of(c, dims, 8);
          CHECK(piece >= 0 && piece + 8 <= pairs);
          if (c < dims) CHECK(piece == at);
        }
      }
  return 0;
}
