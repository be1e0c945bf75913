// The dispatch rules of the linear's products behind a C interface, for tests.
#include <stddef.h>

#include "linear_rules.hpp"

extern "C" {
// height, width, slices, per, mid of the plan
void rule_product(int bf16, int tiles_ok, int a_along, int b_along, long long M, long long N, long long K,
                  int cus, int* out) {
  const fs::ProductPlan p = fs::product_plan(bf16, tiles_ok, a_along, b_along, M, N, K, cus);
  out[0] = p.height, out[1] = p.width, out[2] = p.slices, out[3] = p.per, out[4] = p.mid;
}
long long rule_product_ws(int bf16, int a_along, int b_along, long long M, long long N, long long K, int cus) {
  return (long long)fs::product_ws(bf16, a_along, b_along, M, N, K, cus);
}
int rule_tile_operand(unsigned long long base, long long ld, long long row) {
  return fs::tile_operand((uintptr_t)base, ld, row);
}
}
