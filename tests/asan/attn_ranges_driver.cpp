// The ranges of a sequence's keys, as the attention kernels compute them, under
// UndefinedBehaviorSanitizer: they cover all keys once, up to the largest length.
#include <stdint.h>
#include <stdio.h>

#include "attn_launch.h"

int main() {
  const int64_t most = ((int64_t)1 << 31) - 4097;
  long cases = 0, bad = 0;
  for (int64_t keys : {(int64_t)-5, (int64_t)0, (int64_t)1, (int64_t)127, (int64_t)128, (int64_t)129, (int64_t)100000,
                       (int64_t)1431655766, (int64_t)1500000000, (int64_t)2146435067, most - 1, most})
    for (int64_t chunk : {(int64_t)128, (int64_t)256, (int64_t)65536, (int64_t)8384640, (int64_t)715827968,
                          (int64_t)1073739776, (int64_t)1073741824, (int64_t)1431655808, most + 1}) {
      const int64_t want = keys > chunk ? (keys + chunk - 1) / chunk : 1;
      const int got = ssn::key_ranges((int)keys, (int)chunk);
      bad += got != want;
      if (want <= 4096)
        for (int64_t r = 0; r < want; ++r) {
          const int64_t begin = r * chunk, end = begin + chunk < keys ? begin + chunk : keys;
          bad += ssn::range_end((int)begin, (int)chunk, (int)keys) != end;
        }
      ++cases;
    }
  if (bad) {
    fprintf(stderr, "%ld wrong ranges\n", bad);
    return 1;
  }
  printf("key ranges ok (%ld cases)\n", cases);
  return 0;
}
