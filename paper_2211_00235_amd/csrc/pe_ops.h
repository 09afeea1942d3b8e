// What pe_block.hip takes from pe_ops.hip: launches without argument checks, for buffers that the library has laid out itself.
#pragma once
#include <hip/hip_runtime.h>

// 8-bit form of [rows][c], c a multiple of 8, rows 16-byte aligned and without gaps
hipError_t ckpt_pack_launch(hipStream_t st, int dtype, const void* x, void* ckpt, long long rows, int c);
hipError_t ckpt_unpack_launch(hipStream_t st, int dtype, const void* ckpt, void* y, long long rows, int c);
