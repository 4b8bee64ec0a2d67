// Device helpers of the matrix products that stage their operands in LDS:
// direct-to-LDS copies, LDS reads with explicit waits, the workgroup barrier,
// and the order in which workgroups take tiles.
#pragma once
#include "layup_internal.h"

#define LDS_PTR(p) ((__attribute__((address_space(3))) void*)(p))

namespace layup {

template <int N>
struct IntC { static constexpr int value = N; };
template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(IntC<I>{});
    static_for<I + 1, N>(f);
  }
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// One 1 KB block, 16 bytes per lane.  (A function template: the builtin's
// width is checked against the target, and the host pass has none.)
template <int>
__device__ __forceinline__ void copy_block(const char* src, char* lds) {
  __builtin_amdgcn_global_load_lds(src, LDS_PTR(lds), 16, 0, 0);
}

// 64 words, 4 bytes per lane.
template <int>
__device__ __forceinline__ void copy_words(const char* src, char* lds) {
  __builtin_amdgcn_global_load_lds(src, LDS_PTR(lds), 4, 0, 0);
}

// LDS reads are inline assembly with explicit lgkmcnt waits: the compiler
// cannot tell an LDS read apart from the direct-to-LDS copies in flight into
// other stages.  Offsets are immediates.
template <int OFF>
__device__ __forceinline__ u32x4 lds_read_b128(uint32_t a) {
  static_assert(OFF >= 0 && OFF < 65536, "LDS immediate offset");
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(a), "n"(OFF));
  return v;
}

template <int OFF>
__device__ __forceinline__ uint32_t lds_read_b32(uint32_t a) {
  static_assert(OFF >= 0 && OFF < 65536, "LDS immediate offset");
  uint32_t v;
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(a), "n"(OFF));
  return v;
}

// Wait until at most N LDS reads are outstanding (LDS reads return in order).
template <int N>
__device__ __forceinline__ void lgkm_wait() {
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N < 15 ? N : 15));
}

// Make the MFMA that consumes v depend on the preceding wait.
__device__ __forceinline__ void after_wait(u32x4& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void after_wait(uint32_t& v) { asm volatile("" : "+v"(v)); }

// s_waitcnt vmcnt(n), expcnt and lgkmcnt left alone (gfx9 encoding).
#define WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | (7 << 4) | (15 << 8))

// Workgroup barrier without the release fence of __syncthreads(): the fence
// would make the compiler drain every outstanding direct-to-LDS load
// (vmcnt(0)) at each K step; the exact wait is issued by hand before it.
__device__ __forceinline__ void barrier_only() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// The logical work item of a hardware workgroup.  The grid is one dimension
// of n work items, padded to a multiple of 8.  Workgroups are dealt round-robin
// over the 8 XCDs (each with its own L2), so hardware id h runs on XCD h % 8:
// the remap gives every XCD a contiguous range of logical ids, i.e. whole
// bands of tiles of one batch/split that share operand rows.
__device__ __forceinline__ int work_item(int n, int h) {
  return (h & 7) * ((n + 7) >> 3) + (h >> 3);
}

}  // namespace layup
