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

// Rows [begin, end) of sequence b, cut to [0, rows)
struct PromptSpan {
    int begin, end;
};
__device__ __forceinline__ PromptSpan prompt_span(const int32_t* row0, int b, int rows)
{
    const int lo = min(max(row0[b], 0), rows), hi = min(max(row0[b + 1], 0), rows);
    return {lo, max(lo, hi)};
}

// Which unit of work a workgroup has, if sequence b has count(b) units and they are numbered sequence by sequence: the sequence (-1: none,
// there are fewer) and the number within it.  By all lanes of every wavefront alike, 64 sequences at a time.
struct PromptUnit {
    int seq, index;
};
template <typename COUNT>
__device__ __forceinline__ PromptUnit prompt_unit(int unit, int batch, COUNT count)
{
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int n = b0 + lane < batch ? count(b0 + lane) : 0;
        int sum = n;   // up to and with this lane
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(sum, d);
            if (lane >= d) sum += below;
        }
        const int total = __builtin_amdgcn_readlane(sum, 63);
        if (unit < total) {
            const int at = __builtin_ctzll(__ballot(unit < sum));
            return {b0 + at, unit - __builtin_amdgcn_readlane(sum - n, at)};
        }
        unit -= total;
    }
    return {-1, 0};
}

}  // namespace specv
