// Attention of one new word per text over a cache in pages: step.h with a look into the table of pages a step ahead of the rows.
#include "step.h"

namespace w2v {

void launch_step_pages(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) step_any<float, true>(a, st);
    else if (type == ELEM_F16) step_any<_Float16, true>(a, st);
    else step_any<__bf16, true>(a, st);
}

}  // namespace w2v
