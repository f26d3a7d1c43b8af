// CPU check of how an attention in a window is cut (cache_attend_parts): "tiles wholes most alike group" a line, parts a line.
#include "ss_cache.h"

#include <cstdio>

int main() {
  long long tiles, wholes, most;
  int alike, group;
  while (scanf("%lld %lld %lld %d %d", &tiles, &wholes, &most, &alike, &group) == 5)
    printf("%d\n", ss::cache_attend_parts(tiles, wholes, most, alike != 0, group != 0));
  return 0;
}
