// The kernel and splits that the prompt's attention takes for shapes on standard input:
// batch, KV heads, query heads per KV head, head dimension, element size, query rows, keys,
// window, sinks.
#include <stdio.h>

#include "kvec_prefill_plan.h"

int main() {
  kvec::PrefillShape a;
  while (scanf("%d %d %d %d %d %d %d %d %d", &a.batch, &a.H, &a.G, &a.D, &a.esize, &a.q_len, &a.kv_len, &a.window, &a.sinks) == 9) {
    static const char* const names[] = {"rows16", "rows16_keys", "rows32", "rows32_half", "rows32_keys", "rows32_keys4", "few"};
    a.HQ = a.H * a.G;
    const kvec::PfPlan p = kvec::pf_plan(a);
    printf("%s %d\n", names[p.kernel], p.S);
  }
}
