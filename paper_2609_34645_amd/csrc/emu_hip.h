// What the library's device code and its launches share: loads and stores by cache policy, device attributes,
// launch errors. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>

#include "emu_internal.h"

namespace emu {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------------
// device helpers
// ------------------------------------------------------------------------------------------------

// Global-address-space views: table-loaded pointers are generic to the compiler, which would emit
// flat loads; casting to address space 1 gives global_load/store_dwordx4 with a scalar base.
typedef __attribute__((address_space(1))) v4u gv4u;
typedef __attribute__((address_space(1))) uint8_t gu8;

// Cache policies of the kernels' loads and stores (enum Policy). POL_NT and POL_THROUGH load with "nt" (streaming).
// POL_NT also stores with it; POL_THROUGH stores with "sc1 nt", as buffer stores: written through to memory
// as they come, instead of staying in the XCD's L2 until evicted. With as many tiles in flight as the
// reshard needs to cover its tables' latency, write-through holds HBM's read/write mix better: a bare
// 4 KB-tile copy of 8 GB at 8 / 10 resident waves per CU ran at 6.71 / 6.55 TB/s against 6.52 / 6.28 with
// "nt" (6.80 / 6.73 at 6), the 8B reshard at 10 per CU in 4.80 ms against 4.93. Which call takes which:
// emu_launch.cpp.
constexpr int kThroughBits = 2 | 16;  // nt | sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t whole_range(uint8_t* base) {
  return __builtin_amdgcn_make_buffer_rsrc(base, 0, -1, 0x00020000);  // raw, unswizzled, 2^32 - 1 bytes
}

template <int POL>
__device__ __forceinline__ v4u ld16(const uint8_t* base, uint32_t off) {
  const gv4u* p = (const gv4u*)((const gu8*)base + off);
  if constexpr (POL != POL_PLAIN) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int POL>
__device__ __forceinline__ void st16(uint8_t* base, uint32_t off, v4u v) {
  if constexpr (POL == POL_THROUGH) __builtin_amdgcn_raw_buffer_store_b128(v, whole_range(base), off, 0, kThroughBits);
  else if constexpr (POL == POL_NT) __builtin_nontemporal_store(v, (gv4u*)((gu8*)base + off));
  else *(gv4u*)((gu8*)base + off) = v;
}

__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) v2u gv2u;

template <int POL>
__device__ __forceinline__ v2u ld8(const uint8_t* base, uint32_t off) {
  const gv2u* p = (const gv2u*)((const gu8*)base + off);
  if constexpr (POL != POL_PLAIN) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int POL>
__device__ __forceinline__ void st8(uint8_t* base, uint32_t off, v2u v) {
  if constexpr (POL == POL_THROUGH) __builtin_amdgcn_raw_buffer_store_b64(v, whole_range(base), off, 0, kThroughBits);
  else if constexpr (POL == POL_NT) __builtin_nontemporal_store(v, (gv2u*)((gu8*)base + off));
  else *(gv2u*)((gu8*)base + off) = v;
}

// The same at any element (2-byte) address. gfx950 moves 16 bytes per lane from and to any byte address in
// one instruction; lanes that cover a contiguous span cost one more cache line per instruction. A copy of
// 4 GB from a source 2 bytes off ran at 6.51 TB/s, 4 or 8 bytes off at 6.62, to a destination 2 bytes off at
// 6.66, aligned on both sides at 6.68 (each at its best residency from 8 per CU up), so no realignment in
// registers is needed.
typedef v4u v4u_any __attribute__((aligned(2)));
typedef v2u v2u_any __attribute__((aligned(2)));

template <int POL>
__device__ __forceinline__ v4u ld16_any(const uint8_t* base, uint32_t off) {
  const auto* p = (const __attribute__((address_space(1))) v4u_any*)((const gu8*)base + off);
  if constexpr (POL != POL_PLAIN) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int POL>
__device__ __forceinline__ void st16_any(uint8_t* base, uint32_t off, v4u v) {
  auto* p = (__attribute__((address_space(1))) v4u_any*)((gu8*)base + off);
  if constexpr (POL != POL_PLAIN) __builtin_nontemporal_store(v, p);
  else *p = v;
}

template <int POL>
__device__ __forceinline__ v2u ld8_any(const uint8_t* base, uint32_t off) {
  const auto* p = (const __attribute__((address_space(1))) v2u_any*)((const gu8*)base + off);
  if constexpr (POL != POL_PLAIN) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int POL>
__device__ __forceinline__ void st8_any(uint8_t* base, uint32_t off, v2u v) {
  auto* p = (__attribute__((address_space(1))) v2u_any*)((gu8*)base + off);
  if constexpr (POL != POL_PLAIN) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// A device attribute of the current device, cached per device (0 when it cannot be read).
[[maybe_unused]] static int device_attr(hipDeviceAttribute_t attr, int slot) {
  static std::atomic<int> cache[3][64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 0;
  const bool cached = dev >= 0 && dev < 64;
  if (cached) {
    const int v = cache[slot][dev].load(std::memory_order_relaxed);
    if (v > 0) return v;
  }
  int v = 0;
  if (hipDeviceGetAttribute(&v, attr, dev) != hipSuccess || v <= 0) return 0;
  if (cached) cache[slot][dev].store(v, std::memory_order_relaxed);
  return v;
}

[[maybe_unused]] static int device_cus() {
  const int v = device_attr(hipDeviceAttributeMultiprocessorCount, 0);
  return v > 0 ? v : -1;
}

// Kernel launches report through the runtime's per-thread last-error state. An error some earlier
// runtime call left there belongs to that call, which has already returned it: it is dropped before the
// library launches, so that hip_check afterwards sees only the library's own launches.
static void drop_pending_error() { (void)hipGetLastError(); }

static int hip_check(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(EMU_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return EMU_OK;
}

static bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace emu
