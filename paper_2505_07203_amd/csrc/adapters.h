// Low-rank adapters: what the boundary needs of them.
#pragma once
#include "../../include/po.h"
#include "po_internal.h"

namespace po {

size_t adapters_scratch(int dtype, const int32_t* ranks, int K, const po_adapter_rows* seg, int n_seg);
// ranks, scales, seg: host arrays (see po_op_adapters); res may be null or c
void launch_adapters(int dtype, const void* x, const void* a, const void* b, const int32_t* ranks, const float* scales, int width, const void* res,
                     void* c, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, float* t, hipStream_t s);

}  // namespace po
