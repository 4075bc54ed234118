// Shared by the attention kernels: LDS copies and the swizzles of K and V tiles.
#pragma once

#include "device_common.h"

namespace rp {

constexpr float kLazy = 8.f;  // log2 headroom of the lazily updated softmax max
typedef __attribute__((address_space(3))) void lds_void_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// LDS chunk swizzles (16-byte chunks of a K or V row).  K rows are read 16 bytes per lane
// (row = key), so consecutive keys take distinct chunks.  V rows are read with
// ds_read_b64_tr_b16: in each 32-lane half, lane bits 0,1,4 pick the column within a
// 32-column block and bits 2,3 the key within a group of four; XOR-ing the key's low two
// bits into chunk bits 2,3 (D = 128: a row spans all 64 banks) or 1,2 (D = 64: two rows
// do, the key's bit 0 picking the half) makes the 32 lanes of a half hit 64 distinct
// banks.  (Chunk bits 1,2 at D = 128 left one bank bit fixed: half the banks, and the
// LDS bank-conflict counter at 14% of the prefix kernel's cycles.)
template <int D>
__device__ __forceinline__ int kswz(int key) { return D == 128 ? (key & 15) : (key & 7); }
template <int D>
__device__ __forceinline__ int vswz(int key) { return D == 128 ? (key & 3) << 2 : (key & 3) << 1; }

}  // namespace rp
