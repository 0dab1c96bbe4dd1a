// Device helpers for tiles that go from global memory straight into LDS: the
// loads, the waits and barriers that go with them, and transposed reads.
#pragma once

#include "kamera_device.h"

namespace kamera {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* LdsBytes;
typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;

// Memory that no kernel writes while this one runs, at a wave-uniform address: a scalar
// load.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// Offset of a __shared__ object in the workgroup's LDS.
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(LdsBytes)p; }

// 16 bytes a lane from global memory to LDS: lane i's land at `lds` + 16 i (lds
// wave-uniform).  The instructions are written out because the compiler, which
// cannot tell the tile that is being loaded from the one that is being read, would
// wait for all of them before each read of LDS; vm_wait stands where a tile has to
// be there.  No register but m0 is written, and the address registers are read at issue.
__device__ __forceinline__ void load_lds(const uint8_t* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds(uint64_t address, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(address)
               : "memory", "m0");
}

// Until at most N of the wave's loads are under way.
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The workgroup's waves meet, and this wave's reads of LDS are done.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Four rows of 16 neighbouring 16-bit columns, transposed: lane i of a group of 16
// gives the address of row i / 4, columns 4 (i % 4) .. + 3, and receives column i of
// the four rows.
__device__ __forceinline__ bf16x4 read_columns(uint32_t at) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
}
__device__ __forceinline__ bf16x8 read_chunk(uint32_t at) {
  return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)at;
}
__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

constexpr int kMfma = 0x8, kDsRead = 0x100;        // instruction groups of the scheduler

// The order of N products, each of READS operand reads: kAhead products' reads before
// the first one.
template <int N, int READS, int kAhead>
__device__ __forceinline__ void pipeline() {
  __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead * READS, 0);
#pragma unroll
  for (int i = 0; i < N - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kDsRead, READS, 0);
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, kAhead, 0);
}

}  // namespace kamera
