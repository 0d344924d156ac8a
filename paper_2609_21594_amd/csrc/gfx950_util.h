// Device helpers shared by the kernel files: vector types, bfloat16
// conversions, MFMA, direct-to-LDS and transposing LDS accesses, launch timing.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "muon_internal.h"

namespace muon {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// bfloat16 storage: uint16 bit patterns.  Widening is exact; narrowing is
// the hardware conversion (v_cvt_pk_bf16_f32): round to nearest, ties to
// even, NaN stays NaN, overflow to infinity.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float bf16_to_f32(uint16_t h) {
  return __uint_as_float(static_cast<uint32_t>(h) << 16);
}
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
}
// lo | hi << 16, both rounded as above, in one instruction
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<uint16_t>(uint16_t v) { return bf16_to_f32(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float v) { return f32_to_bf16(v); }

// 8 consecutive elements at base + i (16-byte aligned) as fp32, and back
// (bf16 rounded to nearest even).
template <typename T>
__device__ __forceinline__ void load8(const T* base, int64_t i, float out[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4_t raw = *reinterpret_cast<const u32x4_t*>(base + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      out[2 * q] = __uint_as_float(raw[q] << 16);
      out[2 * q + 1] = __uint_as_float(raw[q] & 0xffff0000u);
    }
  } else {
    const float4 a = *reinterpret_cast<const float4*>(base + i);
    const float4 b = *reinterpret_cast<const float4*>(base + i + 4);
    out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w;
    out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* base, int64_t i, const float in[8]) {
  if constexpr (sizeof(T) == 2) {
    u32x4_t raw;
#pragma unroll
    for (int q = 0; q < 4; ++q) raw[q] = pack_bf16x2(in[2 * q], in[2 * q + 1]);
    *reinterpret_cast<u32x4_t*>(base + i) = raw;
  } else {
    *reinterpret_cast<float4*>(base + i) = make_float4(in[0], in[1], in[2], in[3]);
    *reinterpret_cast<float4*>(base + i + 4) = make_float4(in[4], in[5], in[6], in[7]);
  }
}

template <typename T> struct Mma;
template <> struct Mma<uint16_t> {
  __device__ __forceinline__ static void run(const u32x4_t& a, const u32x4_t& b, f32x16_t& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  }
};
template <> struct Mma<float> {
  __device__ __forceinline__ static void run(const u32x4_t& a, const u32x4_t& b, f32x16_t& c) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c,
                                               0, 0, 0);
  }
};

// Byte offset of an LDS object.
__device__ __forceinline__ uint32_t lds_offset(const char* p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)(p)));
}

// Direct global -> LDS load (global_load_lds_dwordx4): lane i writes the 16
// bytes at base + off (base wave-uniform, off a 32-bit lane offset) to LDS
// bytes [lds + 16 i, lds + 16 i + 16); `lds` is wave-uniform.  Issued as
// inline assembly so that the compiler keeps no record of it: the kernel
// waits for these loads explicitly (vmcnt) before the barrier that publishes
// a slab, and the transposing LDS reads of the other stage must not wait for
// them.  M0 is set inside the statement.
__device__ __forceinline__ void load_lds16(const char* base, uint32_t off, uint32_t lds) {
  // (readfirstlane returns int: widen each half as unsigned, never by sign)
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b & 0xffffffffu)));
  const uint64_t bs = (static_cast<uint64_t>(hi) << 32) | static_cast<uint64_t>(lo);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(off), "s"(bs), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}

// The same with 4 bytes a lane (global_load_lds_dword).
__device__ __forceinline__ void load_lds4(const char* base, uint32_t off, uint32_t lds) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b & 0xffffffffu)));
  const uint64_t bs = (static_cast<uint64_t>(hi) << 32) | static_cast<uint64_t>(lo);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :: "v"(off), "s"(bs), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}

// 8 bytes per lane from LDS through the transposing read (ds_read_b64_tr_b16).
__device__ __forceinline__ uint2 tr_read_b64(const char* p) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4i16*)(const_cast<char*>(p)));
  return __builtin_bit_cast(uint2, v);
}

// Brackets one launch with the optional timer.
struct Timed {
  LaunchTimer* t;
  int kind;
  hipStream_t st;
  Timed(LaunchTimer* timer, int k, hipStream_t s) : t(timer), kind(k), st(s) {
    if (t) t->begin(kind, st);
  }
  void done(double flops, double exec_flops, double bytes) {
    if (t) t->end(kind, st, flops, exec_flops, bytes);
  }
};

}  // namespace
}  // namespace muon
