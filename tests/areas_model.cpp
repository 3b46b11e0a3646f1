// compams_areas.h against the bytes themselves, for every pair of small areas.
#include <stdio.h>

#include <vector>

#include "compams_areas.h"

using compams::Area;

int main() {
  const char* const base = reinterpret_cast<const char*>(1 << 20);
  std::vector<Area> all;
  for (int64_t rows = 0; rows <= 4; ++rows)
    for (int64_t bytes = 0; bytes <= 4; ++bytes)
      for (int64_t ld = rows <= 1 ? 0 : bytes ? bytes : 1; ld <= (rows <= 1 ? 0 : 7); ++ld) all.push_back({base, rows, bytes, ld});
  int64_t exact = 0, wrong = 0, cautious = 0;
  for (const Area& a : all)
    for (const Area& b0 : all)
      for (int at = -36; at <= 36; ++at) {
        Area b = b0;
        b.p = base + at;
        bool shared = false;
        for (int64_t i = 0; i < a.rows; ++i)
          for (int64_t j = 0; a.bytes && j < b.rows; ++j)
            shared |= b.bytes && at + j * b.ld < i * a.ld + a.bytes && i * a.ld < at + j * b.ld + b.bytes;
        const bool met = compams::meet(a, b);
        if (met == shared) ++exact;
        // only of two distances may areas be taken to meet that do not
        else if (met && a.rows > 1 && b.rows > 1 && a.ld != b.ld) ++cautious;
        else ++wrong;
      }
  const Area none = {nullptr, 3, 4, 4}, one = {base, 3, 4, 4}, far = {base, INT32_MAX, 1, INT64_C(1) << 33};
  const Area still = {base, 3, 4, 0}, row = {base, 1, 4, 0};  // (rows that are not apart)
  if (!compams::meet(still, row) || !compams::meet(row, still)) ++wrong;
  if (compams::meet(none, one) || compams::meet(one, none) || !compams::meet(far, one) || !compams::meet(one, far)) ++wrong;
  printf("%lld exact, %lld cautious, %lld wrong\n", (long long)exact, (long long)cautious, (long long)wrong);
  return wrong != 0;
}
