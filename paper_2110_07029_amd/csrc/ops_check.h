// Host-side checks of the matrices, lists and scratch memory that callers hand to the
// entry points over label logits (api_logits.hip, api.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/asgd.h"
#include "asgd_kernels.h"

namespace asgd {

asgd_status set_error(asgd_status s, const char* msg);
asgd_status set_error_named(asgd_status s, const char* name, const char* msg);

asgd_status hip_failed(hipError_t e, const char* what);

// Sizes, type, stride and alignment of a matrix (label_rows: it may have as many rows as a model labels).
asgd_status check_matrix(const asgd_matrix* a, const char* name, bool label_rows = false);
// Lists of ids (and values) per row, for rows x cols logits; NULL is fine.
asgd_status check_list(const asgd_csr* a, const char* name, int rows, int cols, bool values);
// The lists as the kernels take them, from row `row0` on.
IdLists list_dev(const asgd_csr* a, int row0);
// The same of an MXFP4 matrix.
asgd_status check_fp4(const asgd_fp4* q, const char* name);
// The rules for rows of `cols` labels, `rows` of them.
asgd_status check_rules(const asgd_logit_rules* r, int rows, int cols);
asgd_status check_temperature(float t);
// The rules as the kernels take them, from row `row0` on.
RankRules rules_dev(const asgd_logit_rules* r, int row0);
// The device memory that the rules name belongs to the current device.
asgd_status check_rules_memory(const asgd_logit_rules* r);

// p is device or managed memory of the current device.
asgd_status check_device(const void* p, const char* name);
// The same for a device that the caller has looked up.
asgd_status check_device_is(int dev, const void* p, const char* name);
asgd_status check_stream(void* hip_stream);
asgd_status check_workspace(const void* ws, size_t have, size_t need);

}  // namespace asgd
