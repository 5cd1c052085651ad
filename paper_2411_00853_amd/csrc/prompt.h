// What the operators on packed prompts (spec_prompt.h) share on the device.
#pragma once

#include "common.h"
#include "q8.h"   // bf16 rounding, loads of eight elements, requests straight into LDS and their waits
#include "../../include/spec_prompt.h"

namespace specv {

typedef __bf16 pr_bf16x8 __attribute__((ext_vector_type(8)));
typedef float pr_floatx4 __attribute__((ext_vector_type(4)));
typedef float pr_floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned pr_uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned pr_uintx4 __attribute__((ext_vector_type(4)));

// Two numbers as bf16, the first one in the low half
__device__ __forceinline__ unsigned pr_pack2(float a, float b)
{
    const q8_bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, v);
}

// Sixteen bytes, at any even address, of an output as long as a prompt: past the L2s, which then keep what is read.  The norm of 4096 x 4096 fp32 (operands
// from memory) 24.6 -> 19.7 us, of bf16 rows 20.8 -> 15.4, the rotary embedding of 6020 rows 84.4 -> 81.  A pass, whose next kernel reads them, hardly
// notices: 8 layers of the 7B shape with 37 tokens 1.021 -> 1.031 ms, 100 1.372 -> 1.362, 300 2.169 -> 2.162, 1000 3.715 -> 3.766, 3328 10.55 both ways.
__device__ __forceinline__ void pr_stream(void* to, const pr_uintx4& v)
{
    typedef pr_uintx4 __attribute__((aligned(2))) Any;
    __builtin_nontemporal_store(v, (Any*)to);
}

// Rows [begin, end) of sequence b, cut to [0, rows)
struct PromptSpan {
    int begin, end;
};
__device__ __forceinline__ PromptSpan prompt_span(const int32_t* row0, int b, int rows)
{
    const int lo = min(max(row0[b], 0), rows), hi = min(max(row0[b + 1], 0), rows);
    return {lo, max(lo, hi)};
}

// n / d for 0 <= n < 2^31, by a product (the compiler's division by a number it does not know is some forty instructions)
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t by) : d(by)
    {
        uint32_t l = 0;
        while (((uint64_t)1 << l) < by) ++l;
        shift = 31 + l;
        mul = (uint32_t)(((uint64_t)1 << shift) / by + 1);   // n (mul / 2^shift - 1 / d) < 2^31 2^-shift <= 1 / d: what is cut off is below a d-th
    }
    __device__ __forceinline__ int div(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};

// The sum over the lanes up to and with each one (by DPP: a chain of six permutations through LDS takes 700 cycles)
__device__ __forceinline__ int wave_scan(int v)
{
#define PR_STEP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false)
    PR_STEP(0x111, 0xf);    // from 1, 2, 4, 8 lanes below within sixteen, then from the last lane of the sixteen, of the half below
    PR_STEP(0x112, 0xf);
    PR_STEP(0x114, 0xf);
    PR_STEP(0x118, 0xf);
    PR_STEP(0x142, 0xa);
    PR_STEP(0x143, 0xc);
#undef PR_STEP
    return v;
}

// Which unit of work a workgroup has, if sequence b has count(b) units: the sequence (-1: none, there are fewer units) and the unit's number within
// it.  Units are numbered sequence by sequence, the last one of each first; by_place: 64 sequences at a time, those with the highest number within
// their sequence first.  By all lanes of every wavefront alike.
struct PromptUnit {
    int seq, index, lane;   // lane: which one has counted the sequence
};
template <typename COUNT>
__device__ __forceinline__ PromptUnit prompt_unit(int unit, int batch, bool by_place, COUNT count)
{
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int n = b0 + lane < batch ? count(b0 + lane) : 0, sum = wave_scan(n);
        const int total = __builtin_amdgcn_readlane(sum, 63);
        if (unit >= total) {
            unit -= total;
            continue;
        }
        if (!by_place) {
            const int at = __builtin_ctzll(__ballot(unit < sum));
            return {b0 + at, __builtin_amdgcn_readlane(sum, at) - 1 - unit, at};
        }
        auto from = [&](int index) { return __builtin_amdgcn_readlane(wave_scan(max(n - index, 0)), 63); };   // units with this number or a higher one
        int lo = 0, hi = 1;     // from(lo) > unit >= from(hi)
        while (from(hi) > unit) {
            lo = hi;
            hi *= 2;
        }
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (from(mid) > unit) lo = mid;
            else hi = mid;
        }
        const int nth = unit - from(hi);            // (by all lanes)
        const uint64_t with = __ballot(n > lo);     // those sequences have a unit of this number, and this many of them come before the lane's
        const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(with >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)with, 0u));
        const int at = __builtin_ctzll(__ballot(n > lo && before == nth));
        return {b0 + at, lo, at};
    }
    return {-1, 0, 0};
}

}  // namespace specv
