// Loads by buffer descriptor, tiles in LDS, barriers, the order of work-groups.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_device.h"

namespace rc {

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ uint32_t lds_u32(const char* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_void*)p));
}

// 16 bytes per lane straight into LDS at M0 + 16 lane; offsets past the record
// count read as zeros.  Counted in vmcnt, in order with the wave's other loads.
__device__ __forceinline__ void dma16(uint32_t lds, uint32_t voff, __amdgpu_buffer_rsrc_t rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, int(bytes), 0x00020000);
}

// 16 bytes; zeros past the record count, and where `in` is false.  Without a branch, so
// that many are in flight.
__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off, bool in) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, int(in ? off : 0xfffffff0u), 0, 0);
}

// Barrier that waits for this wave's LDS accesses but not for its loads in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
}

__device__ __forceinline__ void sched_fence() { __builtin_amdgcn_sched_barrier(0); }

// The hardware deals work-groups round-robin to the 8 XCDs; give each XCD a
// contiguous run of logical tiles, whose operands its L2 then shares.
__device__ __forceinline__ int64_t xcd_block(int64_t bid, int64_t nblk) {
  const int64_t xcd = bid & 7, kx = bid >> 3, per = nblk >> 3, rem = nblk & 7;
  return (xcd < rem) ? xcd * (per + 1) + kx : rem * (per + 1) + (xcd - rem) * per + kx;
}

// Logical tile w of rows x cols: groups of `group` row tiles, rows fastest inside a group.
template <typename Int>
__device__ __forceinline__ void grouped_tile(Int w, Int rows, Int cols, int group, Int& row, Int& col) {
  const Int per_group = group * cols;
  const Int first = w / per_group * group;
  const Int n = min(Int(group), rows - first);
  const Int in = w % per_group;
  row = first + in % n;
  col = in / n;
}

}  // namespace rc
