// The places of the relative position bias's map (csrc/places.h) against the
// definition in 64 bits: small and the largest maps, differences on both sides
// of either end and far beyond, every offset near the ends of its range.
#include <cstdio>

#include "places.h"

int main() {
  const int64_t Rs[] = {0, 1, 2, 128, 4097, (1 << 29) - 1, 1 << 29, (1 << 30) - 5000, (1 << 30) - 1};
  const int64_t far = int64_t{1} << 62;
  long checked = 0;
  for (const int64_t R : Rs) {
    const int64_t firsts[] = {-far - R, -(int64_t{1} << 31), -R - (1 << 30) - 1, -R - (1 << 30), -R - 5000, -R - 1,
                              -R,       -1,                  0,                  R - 5000,        R - 1,     R,
                              R + 1,    R + 5000,            int64_t{1} << 31,   far - R};
    for (const int64_t at : firsts)
      for (int64_t d = -3; d <= 3; ++d)
        for (const int64_t from : {int64_t{0}, int64_t{4090}, int64_t{(1 << 30) - 16}})
          for (int64_t u = from; u < from + 16; ++u) {
            const int64_t first = at + d, rel = first + u;
            const int64_t want = (rel < -R ? -R : rel > R ? R : rel) + R;
            const int64_t got = emb::place(emb::base_of(first, static_cast<int32_t>(R)), static_cast<int32_t>(u),
                                           static_cast<int32_t>(R));
            ++checked;
            if (got != want) {
              std::printf("R %lld, difference %lld + %lld: place %lld, not %lld\n", (long long)R, (long long)first,
                          (long long)u, (long long)got, (long long)want);
              return 1;
            }
          }
  }
  std::printf("ok: %ld places\n", checked);
  return 0;
}
