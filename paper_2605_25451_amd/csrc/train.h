// Shared by the operators of bigmac_train.h.
#pragma once
#include "common.h"
#include "../../include/bigmac_train.h"

namespace bm {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool good_dtype(int dtype) { return dtype == BM_DTYPE_BF16 || dtype == BM_DTYPE_FP32; }

}  // namespace bm
