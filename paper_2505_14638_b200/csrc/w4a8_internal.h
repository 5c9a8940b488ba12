// Host-side helpers that the library's translation units share (defined in w4a8_lib.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace w4a8 {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_device();                 // W4A8_OK on a device of compute capability 10.x
unsigned int* status_word_ptr();    // the device status word of the current device, nullptr on failure
int launch_status();                // W4A8_OK, or W4A8_ERR_CUDA after a failed launch
void count_launch();                // w4a8_launch_count
int sm_count();                     // SMs of the current device, 0 on failure

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn();

}  // namespace w4a8
