// Host interface of the calls over lists of arrays (list_ops.cu, compiled in a unit of its own).
#pragma once

#include "dion_common.cuh"

namespace dion {
namespace list {

// What a call needs of its context.
struct Where {
  int sm_count;
  void* (*scratch)(void* owner, cudaStream_t stream);      // scratch_bytes() for one call, zero at first; only long norms ask for it
  void* owner;
  int* status;            // [0] status bits, [1] cancelled steps
  int64_t* launches;
  cudaStream_t stream;
};

size_t scratch_bytes();

// Loads every kernel (a kernel's first use could otherwise fall into a stream capture).
int configure();

int grad_norm(const Where& w, const dion_grad* list, int count, int norm_type, float max_norm, float* norm_out, float* each_out,
              float* coef_out);
int clip_grads(const Where& w, const dion_grad* list, int count, float max_norm, int norm_type, const float* norms, int num_norms,
               float* norm_out, float* coef_out);
int param_step(const Where& w, bool adamw, const dion_param* list, int count, const dion_rule* rule, float lr);

// The arguments alone (no device is touched).
int check_norm(const dion_grad* list, int count, int norm_type, float max_norm, const float* norm_out, const float* each_out, const float* coef_out);
int check_clip(const dion_grad* list, int count, float max_norm, int norm_type, const float* norms, int num_norms,
               const float* norm_out, const float* coef_out);
int check_step(bool adamw, const dion_param* list, int count, const dion_rule* rule, float lr);

}  // namespace list
}  // namespace dion
