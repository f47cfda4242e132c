// Which form a call of attn_received takes: most, last, requests, KV heads and group's heads a line on stdin, 1 (pairs of blocks) or 0 on stdout.
#include <stdio.h>

#include "span_rules.h"

int main() {
  long long most, last, requests, heads, group;
  while (scanf("%lld %lld %lld %lld %lld", &most, &last, &requests, &heads, &group) == 5) printf("%d\n", hyp::span_received_pairs(most, last, requests, heads, group));
  return 0;
}
