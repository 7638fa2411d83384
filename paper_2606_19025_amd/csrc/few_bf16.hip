// The few-token layer's projections (few.h) on bf16 weights: tiles for up to 16, 32, 48 and 64 tokens.
#include "few.h"

namespace moe {
namespace {
template <int ACT>
void run(const FewArgs& a, hipStream_t s) {
  if (a.T <= 16) few_launch<bf16_t, false, ACT, 1>(a, s);
  else if (a.T <= 32) few_launch<bf16_t, false, ACT, 2>(a, s);
  else if (a.T <= 48) few_launch<bf16_t, false, ACT, 3>(a, s);
  else few_launch<bf16_t, false, ACT, 4>(a, s);
}
}  // namespace

void run_few_bf16(const FewArgs& a, bool swiglu, hipStream_t s) {
  swiglu ? run<MOE_ACT_SWIGLU>(a, s) : run<MOE_ACT_SILU>(a, s);
}

}  // namespace moe
