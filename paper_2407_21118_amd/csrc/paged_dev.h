// Device-side helpers of the kernels for attention over a paged latent cache.
#pragma once

#include "paged.h"

namespace palu {

namespace {

constexpr float kKeyScale = 0.125f;
template <int N> struct IntC { static constexpr int value = N; };

template <typename T> __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c);
template <> __device__ __forceinline__ float4v mma<F16>(uint4v a, uint4v b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4v mma<BF16>(uint4v a, uint4v b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// two float32 numbers as a pair of 16-bit ones hi, and what the rounding left as another, lo
template <typename T> __device__ __forceinline__ uint32_t pack2(float x, float y);
template <> __device__ __forceinline__ uint32_t pack2<F16>(float x, float y) {
  return __builtin_bit_cast(uint32_t, half2v{(_Float16)x, (_Float16)y});
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <> __device__ __forceinline__ uint32_t pack2<BF16>(float x, float y) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}
// x less the 16-bit number in the low half of h.  As a multiply-add it takes a float16 operand as it is.
template <typename T> __device__ __forceinline__ float less(float x, uint32_t h, float minus_one = -1.f) {
  return __builtin_fmaf(T::to_float((uint16_t)h), minus_one, x);
}
template <typename T> __device__ __forceinline__ void split2(float x, float y, uint32_t* hi, uint32_t* lo) {
  uint32_t h = pack2<T>(x, y);
  asm("" : "+v"(h));           // lo has to be measured from these very bits: where x is a product, the compiler may round it to hi in one step and
  *hi = h;                     // take the conversion of the float32 product, another number now and then, for hi's value
  *lo = pack2<T>(less<T>(x, h), less<T>(y, h >> 16));
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 16 (4) bytes per lane from g to LDS byte m0 + 16 (4) * lane; counted by vmcnt, without a register
__device__ __forceinline__ void load_to_lds(const void* g, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(m0), "v"(g) : "memory");
}
__device__ __forceinline__ void load_to_lds4(const void* g, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(m0), "v"(g) : "memory");
}
// waits until at most n (rounded down to what is listed) of this wavefront's vector-memory operations are outstanding
__device__ __forceinline__ void wait_vm(int n) {
  if (n >= 36) asm volatile("s_waitcnt vmcnt(36)" ::: "memory");
  else if (n >= 30) asm volatile("s_waitcnt vmcnt(30)" ::: "memory");
  else if (n >= 27) asm volatile("s_waitcnt vmcnt(27)" ::: "memory");
  else if (n >= 24) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
  else if (n >= 20) asm volatile("s_waitcnt vmcnt(20)" ::: "memory");
  else if (n >= 18) asm volatile("s_waitcnt vmcnt(18)" ::: "memory");
  else if (n >= 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else if (n >= 14) asm volatile("s_waitcnt vmcnt(14)" ::: "memory");
  else if (n >= 12) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
  else if (n >= 10) asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
  else if (n >= 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if (n >= 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else if (n == 5) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
  else if (n == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
  else if (n == 3) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
  else if (n == 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else if (n == 1) asm volatile("s_waitcnt vmcnt(1)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
// the larger of x over the four lanes that differ in lane bits 4 and 5
__device__ __forceinline__ float max_of_4(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1])));
  auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
// This wavefront's LDS operations are done, and so are the other wavefronts'; loads to LDS go on.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace

}  // namespace palu
