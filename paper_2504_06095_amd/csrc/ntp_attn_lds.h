// Building blocks of the attention kernels over the paged cache: exchanges between the lanes of a wavefront, DMA into the LDS, LDS reads as inline assembly with their waits (not part
// of the ABI).
#ifndef NTP_ATTN_LDS_H_
#define NTP_ATTN_LDS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "ntp_gemm_kernels.h"
#include "ntp_gemm_ring.h"

namespace ntp_attn {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum / sum over the four lanes l % 16 + {0, 16, 32, 48}, left in all four: the 16-lane rows, then the halves trade places in registers.
template <typename F>
__device__ __forceinline__ float over_rows(float v, F&& f) {
  {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    v = f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
  }
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  return f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}

// `bytes` bytes at p; what lies behind them reads as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t view(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
__device__ __forceinline__ void dma_16(__amdgpu_buffer_rsrc_t rs, unsigned char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ntp_gemm::lds_void*)dst, 16, off, 0, 0, 2);
}
// The same for what other workgroups read too: it stays in the caches.
__device__ __forceinline__ void dma_16_shared(__amdgpu_buffer_rsrc_t rs, unsigned char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ntp_gemm::lds_void*)dst, 16, off, 0, 0, 0);
}
// All but the last N vector memory instructions have finished.
template <int N>
__device__ __forceinline__ void dma_left() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// What was loaded is there: the compiler's own wait for it stands here and not in a loop, where it would take in the DMA that is in flight.
template <typename V>
__device__ __forceinline__ void arrived(V& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
}

template <int OFF>
__device__ __forceinline__ u32x4 lds_b128(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x4{};
#else
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
template <int OFF>
__device__ __forceinline__ u32x2 lds_tr_b64(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x2{};
#else
  u32x2 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
template <int OFF>
__device__ __forceinline__ u32x2 lds_b64(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x2{};
#else
  u32x2 v;
  asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
// 8-bit elements: of 16 lanes two each name a row's 16, lane l gets the eight rows' element l.
template <int OFF>
__device__ __forceinline__ u32x2 lds_tr8_b64(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x2{};
#else
  u32x2 v;
  asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
// The reads requested before have arrived: every later use of their registers depends on this wait.
template <int N, typename V>
__device__ __forceinline__ void lds_reads_done(V (&r)[N]) {
  static_assert(N % 8 == 0, "");
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(0)"
               : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]), "+v"(r[4]), "+v"(r[5]), "+v"(r[6]), "+v"(r[7])
               :
               : "memory");
#pragma unroll
  for (int i = 8; i < N; i += 8)
    asm volatile("" : "+v"(r[i]), "+v"(r[i + 1]), "+v"(r[i + 2]), "+v"(r[i + 3]), "+v"(r[i + 4]), "+v"(r[i + 5]), "+v"(r[i + 6]), "+v"(r[i + 7]) : : "memory");
#endif
}

// The same for reads whose wait stood in the statement before, and with at most N later reads still in flight.
template <typename V>
__device__ __forceinline__ void lds_reads_tied(V (&r)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]), "+v"(r[4]), "+v"(r[5]), "+v"(r[6]), "+v"(r[7]) : : "memory");
#endif
}
template <int N, typename V>
__device__ __forceinline__ void lds_reads_left(V (&r)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(%8)"
               : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]), "+v"(r[4]), "+v"(r[5]), "+v"(r[6]), "+v"(r[7])
               : "n"(N)
               : "memory");
#endif
}

template <int... Is, typename F>
__device__ __forceinline__ void unrolled(std::integer_sequence<int, Is...>, F&& f) {
  (f(std::integral_constant<int, Is>{}), ...);
}

// Inclusive sum over the wavefront's lanes: inside rows of 16 lanes, then the rows' last values are passed on.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int sum_upto(int v) {
  v = dpp_add<0x111, 0xf>(v);  // shifted by 1, 2, 4, 8 lanes
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);  // lane 15 of a row to the next one: rows 1 and 3
  v = dpp_add<0x143, 0xc>(v);  // lane 31 to rows 2 and 3
  return v;
}

// Over all lanes of a wavefront, for values of at least 0 (f: their sum or maximum), the same way.
template <int CTRL, int ROWS, typename F>
__device__ __forceinline__ float dpp_with(float v, F&& f) {
  return f(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false)));
}
template <typename F>
__device__ __forceinline__ float over_wave(float v, F&& f) {
  v = dpp_with<0x111, 0xf>(v, f);
  v = dpp_with<0x112, 0xf>(v, f);
  v = dpp_with<0x114, 0xf>(v, f);
  v = dpp_with<0x118, 0xf>(v, f);
  v = dpp_with<0x142, 0xa>(v, f);
  v = dpp_with<0x143, 0xc>(v, f);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

}  // namespace ntp_attn

#endif  // NTP_ATTN_LDS_H_
