// y = residual + act(X W^T + bias) for the rows of prompts.  W in the tile order of spec_pack_weight: 1 KiB holds 16 output features by 32 input
// features as one operand of the 16x16x32 matrix instruction, the four tiles of 128 input features lie together.
//
// W is the instruction's first operand: a lane then holds four neighbouring columns of one row of Y, which the epilogue finishes and stores.
#include "prompt.h"

namespace specv {
namespace {

struct Out {
    void* y;
    const float* bias;
    const void* residual;
    int64_t ld_y, ld_r;
    int r_dtype, y_dtype;
    int N;          // columns of y
    bool whole;     // every group of four columns is there and aligned
};

template <int ACT>
__device__ __forceinline__ float activate(float v)
{
    if (ACT == SPEC_ACT_RELU) return v < 0.f ? 0.f : v;
    if (ACT == SPEC_ACT_GELU) return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    if (ACT == SPEC_ACT_SILU || ACT == SPEC_ACT_SWIGLU) return v / (1.f + expf(-v));
    return v;
}

// Row m, columns n .. n + 3: v is the product, up its other half (SPEC_ACT_SWIGLU)
template <int ACT>
__device__ __forceinline__ void finish(const Out& o, int64_t m, int n, pr_floatx4 v, pr_floatx4 up)
{
    if (n >= o.N) return;
    if (o.whole) {
        if (o.bias) v += *reinterpret_cast<const pr_floatx4*>(o.bias + n);
        if (ACT == SPEC_ACT_SWIGLU && o.bias) up += *reinterpret_cast<const pr_floatx4*>(o.bias + o.N + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = activate<ACT>(v[i]) * (ACT == SPEC_ACT_SWIGLU ? up[i] : 1.f);
        if (o.residual) {
            if (o.r_dtype == SPEC_DTYPE_FP32) v += *reinterpret_cast<const pr_floatx4*>((const float*)o.residual + m * o.ld_r + n);
            else {
                const pr_uintx2 r = *reinterpret_cast<const pr_uintx2*>((const uint16_t*)o.residual + m * o.ld_r + n);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
            }
        }
        if (o.y_dtype == SPEC_DTYPE_FP32) *reinterpret_cast<pr_floatx4*>((float*)o.y + m * o.ld_y + n) = v;
        else *reinterpret_cast<pr_uintx2*>((uint16_t*)o.y + m * o.ld_y + n) = (pr_uintx2){pr_pack2(v[0], v[1]), pr_pack2(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= o.N) break;
        float f = v[i], u = up[i];
        if (o.bias) f += o.bias[n + i];
        if (ACT == SPEC_ACT_SWIGLU && o.bias) u += o.bias[o.N + n + i];
        f = activate<ACT>(f) * (ACT == SPEC_ACT_SWIGLU ? u : 1.f);
        const int64_t r = m * o.ld_r + n + i, t = m * o.ld_y + n + i;
        if (o.residual) f += o.r_dtype == SPEC_DTYPE_FP32 ? ((const float*)o.residual)[r] : q8_widen(((const uint16_t*)o.residual)[r]);
        if (o.y_dtype == SPEC_DTYPE_FP32) ((float*)o.y)[t] = f;
        else ((uint16_t*)o.y)[t] = q8_round_bf16(f);
    }
}

// A 16 RT x 16 CT block of products (column tile j of a wavefront: columns 16 j of W)
template <int ACT, int RT, int CT>
__device__ __forceinline__ void finish_block(const Out& o, const pr_floatx4 (&acc)[RT][CT], int m0, int j0, int M)
{
    const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int a = 0; a < RT; ++a) {
        const int m = m0 + 16 * a + r16;
        if (m >= M) continue;
        if constexpr (ACT == SPEC_ACT_SWIGLU) {
#pragma unroll
            for (int b = 0; b < CT; b += 2) finish<ACT>(o, m, (j0 + b) * 8 + 4 * g, acc[a][b], acc[a][b + 1]);
        } else {
#pragma unroll
            for (int b = 0; b < CT; ++b) finish<ACT>(o, m, (j0 + b) * 16 + 4 * g, acc[a][b], acc[a][b]);
        }
    }
}

__device__ __forceinline__ pr_floatx4 mfma(pr_bf16x8 w, pr_bf16x8 x, pr_floatx4 d) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, d, 0, 0, 0); }

constexpr int TILE = 1024;   // bytes of a 16 x 32 tile of W

// ---- many rows: the matrix cores ----------------------------------------------------------------------------------------
//
// WR x WC wavefronts take 16 WR RT rows by 16 WC CT columns.  A stage holds 64 columns of K of both operands; S stages are under way or in use,
// fetched straight into LDS.  W's tiles are in operand order.  X's rows are 128 bytes, the 16-byte pieces of row n in the order piece ^ (n & 7):
// eight lanes fetch a whole line of memory, and the eight lanes of an LDS cycle read eight different groups of banks.
template <int ACT, int WR, int WC, int RT, int CT, int S>
__global__ void __launch_bounds__(64 * WR * WC, WR * WC == 8 ? 2 : 1) tiled_kernel(const uint16_t* __restrict__ x, const uint8_t* __restrict__ w, int64_t ld_x, int M, int K, int n_tiles, int row_blocks,
                                                      int col_blocks, Out out)
{
    constexpr int W = WR * WC, BR = WR * RT, BC = WC * CT;     // row and column tiles of the workgroup
    constexpr int KIB = 2 * (BR + BC), U = (KIB + W - 1) / W;  // KiB of a stage, requests of a wavefront for it
    static_assert(KIB % W == 0, "every wavefront has as many requests");
    static_assert(S * KIB <= 160, "LDS");
    __shared__ __attribute__((aligned(16))) char lds[S * KIB * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int wr = wave / WC, wc = wave % WC;
    // The row blocks of a column block follow each other on one XCD: its L2 has W once
    const int total = row_blocks * col_blocks, xcd = blockIdx.x & 7, each = total >> 3, more = total & 7;
    const int id = xcd * each + min(xcd, more) + (blockIdx.x >> 3);
    const int m0 = (id % row_blocks) * BR * 16, j0 = (id / row_blocks) * BC;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const int n_kb = K >> 5, n_stages = (n_kb + 1) >> 1;

    // KiB q of a stage: W's 2 BC tiles (column tile q / 2, block q % 2 of 32), then eight rows of X each.  Rows and columns beyond the end are the
    // last ones again (never stored); beyond K the pieces of X are the first ones again (never multiplied).
    uint32_t x_off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int q = W * u + wave, row = m0 + 8 * (q - 2 * BC) + (lane >> 3);
        x_off[u] = q < 2 * BC ? 0 : (uint32_t)(min(row, M - 1) - m0) * (uint32_t)(2 * ld_x);
    }
    const uint32_t piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const char* const xb = (const char*)(x + (size_t)m0 * ld_x);
    auto fetch = [&](int stage, int slot) {
        const uint8_t* wb = w + ((size_t)(stage >> 1) * n_tiles + j0) * (4 * TILE) + (stage & 1) * (2 * TILE);
        const char* xs = xb + (size_t)stage * 128;
        const uint32_t p = (uint32_t)stage * 128 + piece < (uint32_t)K * 2 ? piece : piece & 63;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = W * u + wave;
            const uint32_t to = lds0 + (slot * KIB + q) * 1024;
            if (q < 2 * BC) q8_fetch_lds(wb, (uint32_t)min(q / 2, n_tiles - 1 - j0) * (4 * TILE) + (q & 1) * TILE + lane * 16, to);
            else q8_fetch_lds(xs, x_off[u] + p, to);
        }
    };
    pr_floatx4 acc[RT][CT];
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int b = 0; b < CT; ++b) acc[a][b] = (pr_floatx4){0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < min(S - 1, n_stages); ++s) fetch(s, s);
    int slot = 0;
    for (int s = 0; s < n_stages; ++s) {
        if (s + S - 1 <= n_stages) q8_wait_fetches<(S - 2) * U>();
        else q8_wait_fetches<0>();
        q8_barrier();
        if (s + S - 1 < n_stages) fetch(s + S - 1, slot == 0 ? S - 1 : slot - 1);
        const char* base = lds + slot * KIB * 1024;
        const char* wl = base + wc * CT * 2 * TILE + lane * 16;
        const char* xl = base + (2 * BC + wr * RT * 2) * 1024 + r16 * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (2 * s + h >= n_kb) break;
            pr_bf16x8 wf[CT], xf[RT];
#pragma unroll
            for (int b = 0; b < CT; ++b) wf[b] = *reinterpret_cast<const pr_bf16x8*>(wl + (2 * b + h) * TILE);
#pragma unroll
            for (int a = 0; a < RT; ++a) xf[a] = *reinterpret_cast<const pr_bf16x8*>(xl + a * 2048 + (((4 * h + g) ^ (r16 & 7)) * 16));
#pragma unroll
            for (int a = 0; a < RT; ++a)
#pragma unroll
                for (int b = 0; b < CT; ++b) acc[a][b] = mfma(wf[b], xf[a], acc[a][b]);
        }
        slot = slot == S - 1 ? 0 : slot + 1;
        q8_wait_lds();
    }
    finish_block<ACT, RT, CT>(out, acc, m0 + wr * RT * 16, j0 + wc * CT, M);
}

// ---- few rows: the stream of W ------------------------------------------------------------------------------------------
//
// A workgroup takes 16 RT rows by 16 NT columns; its wavefronts share out K by 128 columns and add their sums up in LDS.  Both operands go
// straight into registers, the next 128 columns' while this one's products run.
template <int ACT, int RT, int NT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) skinny_kernel(const uint16_t* __restrict__ x, const uint8_t* __restrict__ w, int64_t ld_x, int M, int K, int n_tiles, Out out)
{
    __shared__ pr_floatx4 part[WAVES][RT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int j0 = blockIdx.x * NT, m0 = blockIdx.y * (16 * RT);
    const int n_kb = K >> 5, n_groups = (n_kb + 3) >> 2;
    pr_floatx4 acc[RT][NT];
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) acc[a][b] = (pr_floatx4){0.f, 0.f, 0.f, 0.f};
    const uint16_t* xr[RT];
#pragma unroll
    for (int a = 0; a < RT; ++a) xr[a] = x + (size_t)min(m0 + 16 * a + r16, M - 1) * ld_x + 8 * g;
    for (int q = wave; q < n_groups; q += WAVES) {
        pr_uintx4 wv[NT][4], xv[RT][4];
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                wv[b][k] = __builtin_nontemporal_load(
                    reinterpret_cast<const pr_uintx4*>(w + ((size_t)q * n_tiles + min(j0 + b, n_tiles - 1)) * (4 * TILE) + k * TILE + lane * 16));
#pragma unroll
        for (int a = 0; a < RT; ++a)
#pragma unroll
            for (int k = 0; k < 4; ++k) xv[a][k] = *reinterpret_cast<const pr_uintx4*>(xr[a] + 32 * min(4 * q + k, n_kb - 1));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (4 * q + k >= n_kb) break;
#pragma unroll
            for (int a = 0; a < RT; ++a)
#pragma unroll
                for (int b = 0; b < NT; ++b)
                    acc[a][b] = mfma(__builtin_bit_cast(pr_bf16x8, wv[b][k]), __builtin_bit_cast(pr_bf16x8, xv[a][k]), acc[a][b]);
        }
    }
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) part[wave][a * NT + b][lane] = acc[a][b];
    __syncthreads();
    // the wavefronts take turns at the blocks (gate and up tile together)
    constexpr int STEP = ACT == SPEC_ACT_SWIGLU ? 2 : 1;
    for (int i = wave * STEP; i < RT * NT; i += WAVES * STEP) {
        pr_floatx4 v[STEP];
#pragma unroll
        for (int t = 0; t < STEP; ++t) {
            v[t] = part[0][i + t][lane];
            for (int k = 1; k < WAVES; ++k) v[t] += part[k][i + t][lane];
        }
        const int m = m0 + 16 * (i / NT) + r16;
        if (m < M) finish<ACT>(out, m, STEP == 2 ? (j0 + i % NT) * 8 + 4 * g : (j0 + i % NT) * 16 + 4 * g, v[0], v[STEP - 1]);
    }
}

struct Call {
    const uint16_t* x;
    const uint8_t* w;
    int64_t ld_x;
    int M, K, n_tiles;
    Out out;
    hipStream_t s;
};

template <int ACT, int RT, int NT, int WAVES>
void launch_skinny(const Call& c)
{
    hipLaunchKernelGGL((skinny_kernel<ACT, RT, NT, WAVES>), dim3((c.n_tiles + NT - 1) / NT, (c.M + 16 * RT - 1) / (16 * RT)), dim3(64 * WAVES), 0, c.s, c.x,
                       c.w, c.ld_x, c.M, c.K, c.n_tiles, c.out);
}

template <int ACT, int WR, int WC, int RT, int CT, int S>
void launch_tiled(const Call& c)
{
    constexpr int BR = WR * RT, BC = WC * CT;
    const int row_blocks = (c.M + 16 * BR - 1) / (16 * BR), col_blocks = (c.n_tiles + BC - 1) / BC;
    hipLaunchKernelGGL((tiled_kernel<ACT, WR, WC, RT, CT, S>), dim3(row_blocks * col_blocks), dim3(64 * WR * WC), 0, c.s, c.x, c.w, c.ld_x, c.M, c.K, c.n_tiles,
                       row_blocks, col_blocks, c.out);
}

template <int ACT>
void launch(const Call& c)
{
    constexpr int NT = ACT == SPEC_ACT_SWIGLU ? 2 : 1;
    if (c.M <= 16) launch_skinny<ACT, 1, NT, 8>(c);
    else if (c.M <= 32) launch_skinny<ACT, 2, NT, 8>(c);
    else if (c.M <= 64) launch_skinny<ACT, 4, NT, 8>(c);
    else if (c.M <= 128) launch_tiled<ACT, 2, 4, 2, 2, 4>(c);
    else launch_tiled<ACT, 2, 4, 8, 4, 2>(c);
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_prompt_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t activation)
{
    return 0;
}

extern "C" int spec_prompt_gemm(const void* x, int64_t ld_x, const void* w_packed, const spec_prompt_epilogue* epilogue, void* y, int32_t y_dtype,
                                int64_t ld_y, int32_t M, int32_t N, int32_t K, void* workspace, size_t workspace_bytes, void* stream)
{
    static const spec_prompt_epilogue none{};
    const spec_prompt_epilogue& e = epilogue ? *epilogue : none;
    if (M < 0 || N <= 0 || K <= 0) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: M = %d, N = %d, K = %d", M, N, K);
    if (e.activation < SPEC_ACT_NONE || e.activation > SPEC_ACT_SWIGLU)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: unknown activation %d", e.activation);
    if (!q8_dtype(y_dtype) || (e.residual && !q8_dtype(e.residual_dtype)))
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: unknown type %d", q8_dtype(y_dtype) ? e.residual_dtype : y_dtype);
    const bool swiglu = e.activation == SPEC_ACT_SWIGLU;
    if (K % 32) return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: K = %d is not a multiple of 32", K);
    if (swiglu && N % 16) return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: N = %d of a gate and up matrix is not a multiple of 16", N);
    if (N > (1 << 23) || K > (1 << 22)) return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: N = %d, K = %d, at most %d and %d", N, K, 1 << 23, 1 << 22);
    if (ld_x < K || ld_x % 8 || ld_x > SPEC_PROMPT_MAX_LD)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: rows of x %lld elements apart (at least %d, a multiple of 8, at most %d)", (long long)ld_x, K,
                    SPEC_PROMPT_MAX_LD);
    if (ld_y < N || (e.residual && e.ld_residual < N))
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: rows of %d columns are %lld elements apart", N, (long long)(ld_y < N ? ld_y : e.ld_residual));
    if (!M) return SPEC_OK;
    if (!x || !w_packed || !y) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: null pointer");
    if (((uintptr_t)x | (uintptr_t)w_packed | (uintptr_t)workspace) & 15)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: x, w_packed and the workspace have to be 16-byte aligned");
    const size_t ys = y_dtype == SPEC_DTYPE_FP32 ? 4 : 2, rs = e.residual_dtype == SPEC_DTYPE_FP32 ? 4 : 2;
    if ((uintptr_t)y % ys || (uintptr_t)e.bias % 4 || (e.residual && (uintptr_t)e.residual % rs))
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: y, bias and residual have to be aligned as their elements");
    if (e.residual == y && (e.residual_dtype != y_dtype || e.ld_residual != ld_y))
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_gemm: the residual is y, but not of its type and ld");
    const int n_out = swiglu ? 2 * N : N;
    const int n_tiles = (n_out + 15) / 16;
    const bool whole = N % 4 == 0 && ld_y % 4 == 0 && (uintptr_t)y % (4 * ys) == 0 && (uintptr_t)e.bias % 16 == 0 &&
                       (!e.residual || (e.ld_residual % 4 == 0 && (uintptr_t)e.residual % (4 * rs) == 0));
    const Call c{(const uint16_t*)x, (const uint8_t*)w_packed, ld_x, M, K, n_tiles,
                 Out{y, e.bias, e.residual, ld_y, e.ld_residual, e.residual_dtype, y_dtype, N, whole}, (hipStream_t)stream};
    if ((int64_t)((M + 15) / 16) * n_tiles > (int64_t)1 << 30 || M > (1 << 26))
        return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: %d rows of %d columns are too many", M, N);
    switch (e.activation) {
    case SPEC_ACT_NONE: launch<SPEC_ACT_NONE>(c); break;
    case SPEC_ACT_RELU: launch<SPEC_ACT_RELU>(c); break;
    case SPEC_ACT_GELU: launch<SPEC_ACT_GELU>(c); break;
    case SPEC_ACT_SILU: launch<SPEC_ACT_SILU>(c); break;
    default: launch<SPEC_ACT_SWIGLU>(c); break;
    }
    SPECV_LAUNCH_CHECK("spec_prompt_gemm");
    return SPEC_OK;
}
