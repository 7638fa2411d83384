// The few-token layer's projections (few.h) on fp32 weights: tiles for up to 16 tokens, or for all.
#include "few.h"

namespace moe {
namespace {
template <int ACT>
void run(const FewArgs& a, hipStream_t s) {
  if (a.T <= 16) few_launch<float, false, ACT, 1>(a, s);
  else few_launch<float, false, ACT, 4>(a, s);
}
}  // namespace

void run_few_f32(const FewArgs& a, bool swiglu, hipStream_t s) {
  swiglu ? run<MOE_ACT_SWIGLU>(a, s) : run<MOE_ACT_SILU>(a, s);
}

}  // namespace moe
