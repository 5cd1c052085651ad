// Rows to 8 bits (e4m3) with a scale for each row and 128 columns: plain, behind SwiGLU, and behind the residual
// addition and RMSNorm of a decoder layer.
//
//     s = max(amax / 448, 2^-126) over a block,  q = e4m3(y / s)
//
// Bound by HBM (by the launch for few rows): every element is read and written once, and the seven bytes of a column of a bf16
// residual row (x, delta and the sum, 8 bits) leave no room for a second pass.  A thread takes eight consecutive columns, sixteen
// threads a block of 128: its largest magnitude is a maximum over sixteen lanes, and the eight bytes of a thread are one store.
// y / s is y times the rounded 1 / s: at most a unit of fp32's last place beside the quotient, 2^-20 of an e4m3 step.
#include "q8.h"

namespace specv {
namespace {

// The maximum over the sixteen lanes of a block, as the bits of a magnitude: a NaN's exceed an infinity's, and both
// exceed any number's, so neither is lost in it.
__device__ __forceinline__ unsigned block_max(unsigned v)
{
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) v = max(v, (unsigned)__shfl_xor((int)v, d));
    return v;
}

// y[8] of one thread -> its bytes; returns the scale of the block
__device__ __forceinline__ float quantise(const float* y, q8_uintx2* bytes)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
    float s = __uint_as_float(block_max(top)) / Q8_MAX;
    s = s < Q8_TINY ? Q8_TINY : s;
    const float r = 1.f / s;
    (*bytes)[0] = q8_pack4(y[0] * r, y[1] * r, y[2] * r, y[3] * r);
    (*bytes)[1] = q8_pack4(y[4] * r, y[5] * r, y[6] * r, y[7] * r);
    return s;
}

// Eight columns from col on, zero beyond cols
template <typename T>
__device__ __forceinline__ void load_cols(const T* row, int col, int cols, float* v)
{
    if (col + 8 <= cols) {
        q8_load8(row + col, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? q8_widen(row[col + i]) : 0.f;
}

constexpr int TPB = 256;

// blockIdx.x: 256 threads of eight columns of a row, blockIdx.y: the row.  No thread waits for another one's load but the fifteen of its
// block, so that many short workgroups keep the memory busy: SwiGLU of 48 x 11008 bf16 3.3 us (launch), of 1333 x 5540 fp32 13 us, 66 MB
// at 5.1 TB/s.
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(TPB) rows_kernel(const T* __restrict__ x, int64_t ld, uint8_t* __restrict__ q, float* __restrict__ scales,
                                                   int rows, int cols, int kp)
{
    const int row = blockIdx.y, col = (blockIdx.x * TPB + threadIdx.x) * 8;
    if (col >= kp) return;   // whole blocks: kp is a multiple of 128
    const T* xr = x + (size_t)row * ld;
    float y[8];
    load_cols(xr, col, cols, y);
    if (SWIGLU) {
        float u[8];
        load_cols(xr + cols, col, cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] / (1.f + expf(-y[i])) * u[i];
    }
    q8_uintx2 bytes;
    const float s = quantise(y, &bytes);
    *reinterpret_cast<q8_uintx2*>(q + (size_t)row * kp + col) = bytes;
    if ((threadIdx.x & 15) == 0) scales[(size_t)(col >> 7) * rows + row] = s;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v);
template <>
__device__ __forceinline__ void store8(float* p, const float* v)
{
    Q8Eight<float> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = v[i];
    *reinterpret_cast<Q8Eight<float>*>(p) = o;
}
template <>
__device__ __forceinline__ void store8(uint16_t* p, const float* v)
{
    Q8Eight<uint16_t> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = q8_round_bf16(v[i]);
    *reinterpret_cast<Q8Eight<uint16_t>*>(p) = o;
}
template <typename T>
__device__ __forceinline__ T narrow(float f)
{
    if constexpr (sizeof(T) == 2) return q8_round_bf16(f);
    else return f;
}

// A workgroup takes a row; a thread holds NV vectors of eight columns, blockDim.x vectors apart, in registers between
// the sum of squares and the rounding.  One vector a thread while there are threads (4096 x 4096 bf16: 31 us, 117 MB at 3.8 TB/s, with one
// as with two; 36 with workgroups that stay and load the next row ahead; which XCD a row goes to makes no difference).  One row of
// 2048: 2.4 us.
template <typename TX, typename TD, int NV>
__global__ void __launch_bounds__(1024) norm_kernel(const TX* x, const TD* __restrict__ delta, const float* __restrict__ gain, int cols, int kp,
                                                    float eps, TX* x_out, uint8_t* __restrict__ q, float* __restrict__ scales, int rows)
{
    __shared__ float wave_sum[16];
    const int row = blockIdx.x, n_waves = blockDim.x >> 6;
    const TX* xr = x + (size_t)row * cols;
    float h[NV][8], ss = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * blockDim.x + threadIdx.x) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k][i] = 0.f;
        if (col < cols) {
            load_cols(xr, col, cols, h[k]);
            if (delta) {
                float d[8];
                load_cols(delta + (size_t)row * cols, col, cols, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[k][i] += d[i];
            }
            if (x_out) {
                TX* o = x_out + (size_t)row * cols + col;
                if (col + 8 <= cols) {
                    store8<TX>(o, h[k]);
                } else if constexpr (NV == 1) {
                    for (int i = 0; i < cols - col; ++i) o[i] = narrow<TX>(h[k][i]);
                } else {   // (an index that is no constant would put all of h into memory: 64 rows of 65536 47 us, 25 this way)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (col + i < cols) o[i] = narrow<TX>(h[k][i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += h[k][i] * h[k][i];
    }
    auto all = [&](float v, auto join) {   // of the workgroup, the same for all threads
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) v = join(v, __shfl_xor(v, d));
        if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
        for (int w = 0; w < n_waves; ++w) v = join(v, wave_sum[w]);
        return v;
    };
    auto add = [](float a, float b) { return a + b; };
    ss = all(ss, add);
    float r = 1.f / sqrtf(ss / (float)cols + eps);
    const float known = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(ss)));   // (the branch is the workgroup's)
    if (!(known <= 0x1.fffffep127f) || (eps == 0.f && known < 0x1p-80f)) {
        // Squares that leave fp32's range: they are those of the row over a power of two near its largest number, if that is one
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(h[k][i]));
        __syncthreads();
        top = all(top, [](float a, float b) { return fmaxf(a, b); });
        const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252);   // (an infinity or a NaN leaves its mark in the sum below)
        const float down = __uint_as_float((unsigned)(254 - e) << 23);
        ss = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[k][i] *= down;
                ss = fmaf(h[k][i], h[k][i], ss);
            }
        __syncthreads();
        ss = all(ss, add);
        r = 1.f / sqrtf(ss / (float)cols + eps * down * down);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * blockDim.x + threadIdx.x) * 8;
        if (col >= kp) continue;
        float g[8], y[8];
        load_cols(gain, col, cols, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = h[k][i] * r * g[i];
        // beyond cols the row is zero whatever r is
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = col + i < cols ? y[i] : 0.f;
        q8_uintx2 bytes;
        const float s = quantise(y, &bytes);
        *reinterpret_cast<q8_uintx2*>(q + (size_t)row * kp + col) = bytes;
        if ((threadIdx.x & 15) == 0) scales[(size_t)(col >> 7) * rows + row] = s;
    }
}

template <typename T, bool SWIGLU>
void launch_rows(const void* x, int64_t ld, int rows, int cols, void* q, float* scales, hipStream_t s)
{
    const int kp = q8_blocks(cols) * SPEC_Q8_BLOCK;
    for (int r0 = 0; r0 < rows; r0 += 65535) {   // the grid's limit in y
        const int n = std::min(65535, rows - r0);
        hipLaunchKernelGGL((rows_kernel<T, SWIGLU>), dim3((kp / 8 + TPB - 1) / TPB, n), dim3(TPB), 0, s,
                           (const T*)x + (size_t)r0 * ld, ld, (uint8_t*)q + (size_t)r0 * kp, scales + r0, rows, cols, kp);
    }
}

template <typename TX, typename TD>
void launch_norm(const void* x, const void* delta, const float* gain, float eps, int rows, int cols, void* x_out, void* q, float* scales,
                 hipStream_t s)
{
    const int kp = q8_blocks(cols) * SPEC_Q8_BLOCK, vecs = kp / 8;
    auto go = [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        const int threads = (((vecs + NV - 1) / NV + 63) / 64) * 64;
        hipLaunchKernelGGL((norm_kernel<TX, TD, NV>), dim3(rows), dim3(threads), 0, s, (const TX*)x, (const TD*)delta, gain, cols, kp, eps,
                           (TX*)x_out, (uint8_t*)q, scales, rows);
    };
    if (vecs <= 512) go(std::integral_constant<int, 1>());
    else if (vecs <= 1024) go(std::integral_constant<int, 2>());
    else if (vecs <= 2048) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 8>());
}

}  // namespace
}  // namespace specv

using namespace specv;

static int check_rows(const char* name, const void* x, int dtype, int rows, int cols, const void* q, const void* scales)
{
    if (rows < 0 || cols <= 0) return fail(SPEC_ERR_INVALID_ARG, "%s: %d rows of %d columns", name, rows, cols);
    if (cols > Q8_MAX_SIZE) return fail(SPEC_ERR_SHAPE, "%s: %d columns, at most %d", name, cols, Q8_MAX_SIZE);
    if (!q8_dtype(dtype)) return fail(SPEC_ERR_INVALID_ARG, "%s: unknown type %d", name, dtype);
    if (rows && (!x || !q || !scales)) return fail(SPEC_ERR_INVALID_ARG, "%s: null pointer", name);
    if ((uintptr_t)q & 15) return fail(SPEC_ERR_INVALID_ARG, "%s: q is not 16-byte aligned", name);
    return SPEC_OK;
}

extern "C" int spec_q8_quantize(const void* x, int32_t x_dtype, int64_t ld, int32_t rows, int32_t cols, void* q, float* scales, void* stream)
{
    if (int rc = check_rows("spec_q8_quantize", x, x_dtype, rows, cols, q, scales)) return rc;
    if (ld < cols) return fail(SPEC_ERR_INVALID_ARG, "spec_q8_quantize: rows of %d columns are %lld elements apart", cols, (long long)ld);
    if (!rows) return SPEC_OK;
    if (x_dtype == SPEC_DTYPE_BF16) launch_rows<uint16_t, false>(x, ld, rows, cols, q, scales, (hipStream_t)stream);
    else launch_rows<float, false>(x, ld, rows, cols, q, scales, (hipStream_t)stream);
    SPECV_LAUNCH_CHECK("rows_kernel");
    return SPEC_OK;
}

extern "C" int spec_q8_swiglu(const void* gate_up, int32_t dtype, int32_t rows, int32_t d_ffn, void* q, float* scales, void* stream)
{
    if (int rc = check_rows("spec_q8_swiglu", gate_up, dtype, rows, d_ffn, q, scales)) return rc;
    if (!rows) return SPEC_OK;
    const int64_t ld = 2 * (int64_t)d_ffn;
    if (dtype == SPEC_DTYPE_BF16) launch_rows<uint16_t, true>(gate_up, ld, rows, d_ffn, q, scales, (hipStream_t)stream);
    else launch_rows<float, true>(gate_up, ld, rows, d_ffn, q, scales, (hipStream_t)stream);
    SPECV_LAUNCH_CHECK("rows_kernel");
    return SPEC_OK;
}

extern "C" int spec_q8_add_rmsnorm(const void* x, int32_t x_dtype, const void* delta, int32_t delta_dtype, const float* gain, float eps,
                                   int32_t rows, int32_t cols, void* x_out, void* q, float* scales, void* stream)
{
    if (int rc = check_rows("spec_q8_add_rmsnorm", x, x_dtype, rows, cols, q, scales)) return rc;
    if (cols > SPEC_Q8_MAX_COLS) return fail(SPEC_ERR_SHAPE, "spec_q8_add_rmsnorm: %d columns, at most %d", cols, SPEC_Q8_MAX_COLS);
    if (delta && !q8_dtype(delta_dtype)) return fail(SPEC_ERR_INVALID_ARG, "spec_q8_add_rmsnorm: unknown type %d", delta_dtype);
    if (!(eps >= 0.f)) return fail(SPEC_ERR_INVALID_ARG, "spec_q8_add_rmsnorm: eps %g", (double)eps);
    if (!rows) return SPEC_OK;
    if (!gain) return fail(SPEC_ERR_INVALID_ARG, "spec_q8_add_rmsnorm: null pointer");
    hipStream_t s = (hipStream_t)stream;
    const bool xb = x_dtype == SPEC_DTYPE_BF16, db = delta && delta_dtype == SPEC_DTYPE_BF16;
    if (xb && db) launch_norm<uint16_t, uint16_t>(x, delta, gain, eps, rows, cols, x_out, q, scales, s);
    else if (xb) launch_norm<uint16_t, float>(x, delta, gain, eps, rows, cols, x_out, q, scales, s);
    else if (db) launch_norm<float, uint16_t>(x, delta, gain, eps, rows, cols, x_out, q, scales, s);
    else launch_norm<float, float>(x, delta, gain, eps, rows, cols, x_out, q, scales, s);
    SPECV_LAUNCH_CHECK("norm_kernel");
    return SPEC_OK;
}
