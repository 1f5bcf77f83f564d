// The window that the cache's kernels get and the tokens that it leaves, from their own header.  Run on the host by test_cache_window_host.py:
// lines of "max_pages page window me" in, "held first" out.
#include <stdio.h>

#include "dsn_cache.cuh"

int main() {
  int max_pages, page, window, me;
  while (scanf("%d %d %d %d", &max_pages, &page, &window, &me) == 4) {
    const int held = dsn_cache_window(window, max_pages, page);
    printf("%d %d\n", held, dsn_cache_first_seen(me, held));
  }
  return 0;
}
