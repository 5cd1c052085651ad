// What the operators on 8-bit numbers (spec_q8.h) share on the device.
#pragma once

#include "common.h"
#include "../../include/spec_q8.h"

namespace specv {

typedef __bf16 q8_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 q8_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 q8_halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 q8_halfx2 __attribute__((ext_vector_type(2)));
typedef float q8_floatx2 __attribute__((ext_vector_type(2)));
typedef float q8_floatx4 __attribute__((ext_vector_type(4)));
typedef int q8_intx4 __attribute__((ext_vector_type(4)));
typedef int q8_intx8 __attribute__((ext_vector_type(8)));
typedef unsigned q8_uintx2 __attribute__((ext_vector_type(2)));

constexpr float Q8_MAX = 448.f;         // largest e4m3 number
constexpr float Q8_TINY = 0x1p-126f;    // smallest scale

constexpr int Q8_MAX_SIZE = 1 << 30;    // of a row or a matrix: places in it, rounded up to whole blocks, are ints

inline int q8_blocks(int cols) { return (cols + SPEC_Q8_BLOCK - 1) / SPEC_Q8_BLOCK; }
inline bool q8_dtype(int t) { return t == SPEC_DTYPE_FP32 || t == SPEC_DTYPE_BF16; }

// Four fp32 numbers to four e4m3 bytes, to nearest even (|v| <= 448 up to rounding, or NaN)
__device__ __forceinline__ unsigned q8_pack4(float a, float b, float c, float d)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

__device__ __forceinline__ float q8_unpack(unsigned byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }

// Eight consecutive elements from any element-aligned address
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Q8Eight {
    T v[8];
};

__device__ __forceinline__ void q8_load8(const float* p, float* v)
{
    const Q8Eight<float> x = *reinterpret_cast<const Q8Eight<float>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x.v[i];
}

__device__ __forceinline__ float q8_widen(uint16_t b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ float q8_widen(float f) { return f; }

__device__ __forceinline__ void q8_load8(const uint16_t* p, float* v)
{
    const Q8Eight<uint16_t> x = *reinterpret_cast<const Q8Eight<uint16_t>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q8_widen(x.v[i]);
}

__device__ __forceinline__ uint16_t q8_round_bf16(float f)
{
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

// The largest of a wavefront's, the same for all lanes (by DPP)
__device__ __forceinline__ unsigned q8_wave_max(unsigned v)
{
#define Q8_STEP(CTRL, ROWS) v = max(v, (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, ROWS, 0xf, false))
    Q8_STEP(0xb1, 0xf);    // neighbours, pairs, halves of a row of sixteen, rows
    Q8_STEP(0x4e, 0xf);
    Q8_STEP(0x141, 0xf);
    Q8_STEP(0x140, 0xf);
    Q8_STEP(0x142, 0xa);
    Q8_STEP(0x143, 0xc);
#undef Q8_STEP
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// 16 bytes (4) per lane straight into LDS, to lds + 16 (4) * lane.  The compiler does not know of the request: wait_fetches.
// (m0 is none of the registers that the compiler hands out, about which it warns; it may set m0 for an instruction of its own.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void q8_fetch_lds(const void* base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void q8_fetch_lds_dword(const void* base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void q8_wait_fetches()   // at most N requests of this wavefront still under way
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void q8_wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void q8_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace specv
