// The shapes of groups at the sizes that a plan lets through, compiled with checks of signed arithmetic: their costs fit 32 bits as long
// as all of them together are below 2^30, and a chunk's place among them is found again.
#include <cstdio>
#include <cstdlib>

#include "attend.cuh"

int main() {
  long long shapes = 0;
  for (int G = 1; G <= 128; G += G < 8 ? 1 : 7)
    for (long long ntok = 2; ntok * G < 1ll << 30; ntok = ntok * 3 + 1)
      for (int pfx = 16; pfx < 1 << 24; pfx = pfx * 5 + 16)
        for (int H = 1; H <= 8; H += 7) {
          const WideShape one((int)ntok, pfx, G, 1);
          const long long cost = (long long)one.tiles * one.sum;
          if (H * cost >= 1ll << 30 || ntok * G * H >= 1ll << 31) continue;
          const int each = (int)((H * cost + 147) / 148) < 2 ? 2 : (int)((H * cost + 147) / 148);
          const WideShape w((int)ntok, pfx, G, (each + 1) / 2);
          if (w.tiles != one.tiles || w.chunks != one.chunks || w.sum != one.sum || (w.stripes - 1) * (long long)w.stripe >= w.tiles || w.stripes * (long long)w.stripe < w.tiles) {
            printf("G %d ntok %lld pfx %d: stripe %d of %d tiles, %d stripes\n", G, ntok, pfx, w.stripe, w.tiles, w.stripes);
            return 1;
          }
          for (int s : {0, w.stripes / 2, w.stripes - 1})
            for (int c : {0, w.whole / 2, w.chunks - 1}) {
              const int x = w.before(s, c), nt = w.tiles_of(s), in = x - s * w.stripe * w.sum;     // as the plan takes it apart
              const int back = in / (nt * 2) < w.whole ? in / (nt * 2) : w.whole;
              if (x < 0 || x >= cost || x / (w.stripe * w.sum) != s || (back < w.chunks - 1 ? back : w.chunks - 1) != c) {
                printf("G %d ntok %lld pfx %d stripe %d chunk %d: %d of %lld\n", G, ntok, pfx, s, c, x, cost);
                return 1;
              }
            }
          ++shapes;
        }
  printf("%lld shapes\n", shapes);
  return shapes < 1000;
}
