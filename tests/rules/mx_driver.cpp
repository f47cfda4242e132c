// Answers questions on how calls of hyp_mx.h are cut, one a line on stdin, one line each on stdout.
#include <stdio.h>
#include <string.h>

#include "mx_rules.h"

int main() {
  char what[16];
  while (scanf("%15s", what) == 1) {
    long long a, b, c, d, e;
    int f, g, h;
    if (!strcmp(what, "token")) {
      if (scanf("%lld %d %lld %lld %lld %lld %d %d", &a, &f, &b, &c, &d, &e, &g, &h) != 8) return 1;
      const hyp::MxTokenPlan t = hyp::mx_token_plan(a, f, b, c, d, e, g, h != 0);
      printf("%d %d %d %d %d\n", t.tiles, t.head_tiles, t.unit, t.units, t.parts);
    } else if (!strcmp(what, "scores")) {
      if (scanf("%lld %lld", &a, &b) != 2) return 1;
      const int turns = hyp::mx_score_turns(a, b);
      printf("%d %d\n", turns, hyp::mx_score_tiles(b, turns));
    } else if (!strcmp(what, "write")) {
      if (scanf("%lld %lld %lld %d", &a, &b, &c, &f) != 4) return 1;
      printf("%lld\n", (long long)hyp::mx_write_tiles(a, b, c, f != 0));
    } else {
      return 1;
    }
  }
  return 0;
}
