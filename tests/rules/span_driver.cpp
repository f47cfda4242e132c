// Answers questions on how calls of hyp_attn.h are cut, one a line on stdin, one line each on stdout.
#include <stdio.h>
#include <string.h>

#include "span_rules.h"

int main() {
  char what[16];
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "prompt")) {
      long long groups, stages, fewest;
      if (scanf("%lld %lld %lld", &groups, &stages, &fewest) != 3) return 1;
      printf("%d\n", hyp::span_prompt_splits(groups, stages, fewest));
    } else if (!strcmp(what, "token")) {
      long long requests, heads, group, most, prefix;
      int waves, stage;
      if (scanf("%lld %lld %lld %lld %lld %d %d", &requests, &heads, &group, &most, &prefix, &waves, &stage) != 7) return 1;
      const hyp::SpanTokenPlan t = hyp::span_token_plan(requests, heads, group, most, prefix, waves, stage);
      printf("%d %d %d %d %d\n", t.pre_wide, t.pre_tiles, t.pre_splits, t.tiles, t.splits);
    } else {
      return 1;
    }
  }
  return 0;
}
