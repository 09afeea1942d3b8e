// What pe_block.hip takes from pe_ops.hip: a launch without argument checks, for buffers that the library has laid out itself.
#pragma once
#include <hip/hip_runtime.h>
#include "../../include/pe.h"

// [rows][c] without gaps into its 8-bit form (pack) or back; c a multiple of 8, both buffers 256-byte aligned.  PE_OK or PE_ERR_HIP.
int ckpt_launch(pe_handle* h, hipStream_t st, bool pack, int dtype, void* x, void* ckpt, long long rows, int c);
