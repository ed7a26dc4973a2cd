// What the C entry points of the attention block's files share (lba_rotary.cu, lba_cache.cu, lba_attention.cu, lba_attention_grad.cu).
#pragma once
#include <cstdint>

#include <cuda_runtime.h>

#include "lba.h"

namespace lba {

int cuda_fail(cudaError_t e);  // lba_api.cu: keeps the code for lba_last_cuda_error
inline int status_of(cudaError_t e) { return e == cudaSuccess ? LBA_OK : cuda_fail(e); }
inline bool half_type(int type) { return type == LBA_TYPE_BF16 || type == LBA_TYPE_F16; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int device_sms();              // lba_api.cu: of the current device

}  // namespace lba
