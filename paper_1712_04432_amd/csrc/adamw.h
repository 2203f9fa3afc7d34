// Internal declarations of the AdamW update (csrc/adamw.hip).
#pragma once

#include "common.h"

namespace imbd {

int64_t adamw_chunks(int64_t n);
void adamw_write_plan(const imbd_adamw_tensor *tensors, int n_tensors, void *plan);
size_t adamw_record_bytes();
size_t adamw_entry_bytes();
int run_adamw(const void *plan, int n_tensors, int64_t chunks, double lr, double beta1, double beta2, double eps,
              float grad_scale, int step, const int32_t *step_dev, hipStream_t s);

}  // namespace imbd
