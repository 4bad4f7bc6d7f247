// What the translation units of the library share: the scratch workspace, the text of the last HIP error,
// the number of compute units.  Defined in gbdt_hist.hip; not exported.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace gbdt_internal __attribute__((visibility("hidden"))) {

int workspace(size_t bytes, hipStream_t s, void** out);  // at least `bytes`, as every call's scratch
size_t workspace_head_bytes();                           // what a registered workspace needs besides
int hip_failed(hipError_t e, const char* what);          // keeps the text, returns GBDT_EHIP
int cu_count();

}  // namespace gbdt_internal
