// y = residual + act(X W^T + bias) for the rows of prompts.  W in the tile order of spec_pack_weight: 1 KiB holds 16 output features by 32 input
// features as one operand of the 16x16x32 matrix instruction, the four tiles of 128 input features lie together.
//
// W is the instruction's first operand: a lane then holds four neighbouring columns of one row of Y, which the epilogue finishes and stores.
#include "prompt.h"

#include <cfloat>

namespace specv {
namespace {

struct Out {
    void* y;
    const float* bias;
    const void* residual;
    int64_t ld_y, ld_r;
    int r_dtype, y_dtype, act;
    int N;          // columns of y
    bool whole;     // every group of four columns is there and aligned
};

template <int ACT>
__device__ __forceinline__ float activate(float v)
{
    if (ACT == SPEC_ACT_RELU) return v < 0.f ? 0.f : v;
    if (ACT == SPEC_ACT_GELU) {
        // erfc(z) = (a1 t + .. + a5 t^5) exp(-z^2), t = 1 / (1 + 0.3275911 z), off by 1.5e-7 at most (Abramowitz and Stegun, 7.1.26).
        // 1333 x 4104 x 2080 with gelu alone 31 us; with the library's erf, before other steps, 40.1 where this took 35.5
        const float z = fabsf(v) * 0.70710678f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
        const float p = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f) * t;
        const float half = 0.5f * p * __builtin_amdgcn_exp2f(z * z * -1.44269504f);
        return v * (v >= 0.f ? 1.f - half : half);
    }
    if (ACT == SPEC_ACT_SILU || ACT == SPEC_ACT_SWIGLU) return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f));
    return v;
}

// Columns n .. n + 3 of y: the products v, with SPEC_ACT_SWIGLU those of the gate rows, and up
struct Four {
    pr_floatx4 v, up;
};
template <bool WHOLE>
__device__ __forceinline__ pr_floatx4 load_bias(const Out& o, int n)
{
    pr_floatx4 b = {0.f, 0.f, 0.f, 0.f};
    if (WHOLE) return *reinterpret_cast<const pr_floatx4*>(o.bias + n);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n % o.N + i < o.N) b[i] = o.bias[n + i];
    return b;
}
// The residual's four numbers as they lie in memory: made floats where they are added, as that has to wait for them
template <bool WHOLE>
__device__ __forceinline__ pr_uintx4 load_residual(const Out& o, int64_t m, int n)
{
    pr_uintx4 r = {0, 0, 0, 0};
    const int64_t at = m * o.ld_r + n;
    if (WHOLE) {
        if (o.r_dtype == SPEC_DTYPE_FP32) return *reinterpret_cast<const pr_uintx4*>((const float*)o.residual + at);
        const pr_uintx2 u = *reinterpret_cast<const pr_uintx2*>((const uint16_t*)o.residual + at);
        r[0] = u[0];
        r[1] = u[1];
        return r;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < o.N) r[i] = o.r_dtype == SPEC_DTYPE_FP32 ? ((const unsigned*)o.residual)[at + i] : (unsigned)((const uint16_t*)o.residual)[at + i] << 16;
    return r;
}
template <bool WHOLE>
__device__ __forceinline__ pr_floatx4 residual_of(const Out& o, const pr_uintx4& r)
{
    const bool pairs = WHOLE && o.r_dtype != SPEC_DTYPE_FP32;
    return (pr_floatx4){__uint_as_float(pairs ? r[0] << 16 : r[0]), __uint_as_float(pairs ? r[0] & 0xffff0000u : r[1]), __uint_as_float(pairs ? r[1] << 16 : r[2]),
                        __uint_as_float(pairs ? r[1] & 0xffff0000u : r[3])};
}
template <bool WHOLE>
__device__ __forceinline__ void store(const Out& o, int64_t m, int n, const pr_floatx4& v)
{
    const int64_t at = m * o.ld_y + n;
    if (WHOLE) {
        if (o.y_dtype == SPEC_DTYPE_FP32) *reinterpret_cast<pr_floatx4*>((float*)o.y + at) = v;
        else *reinterpret_cast<pr_uintx2*>((uint16_t*)o.y + at) = (pr_uintx2){pr_pack2(v[0], v[1]), pr_pack2(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= o.N) break;
        if (o.y_dtype == SPEC_DTYPE_FP32) ((float*)o.y)[at + i] = v[i];
        else ((uint16_t*)o.y)[at + i] = q8_round_bf16(v[i]);
    }
}

// R rows (stride apart in rows) by C groups of four columns, `step` columns apart from n on.  What is read is asked for three rows ahead of its sums
// (1333 x 4104 x 2080 with bias and residual 29.8 us, plain 28.9; lanes that exchange their columns for stores of 16 bytes take 0.5 us off that).
// Whether groups are whole is asked once, here: asked at each access, with gelu, bias and residual 43.1 us where this took 38.4.
template <int ACT, bool WHOLE, int R, int C, typename GET>
__device__ __forceinline__ void finish_as(const Out& o, int m0, int stride, int M, int n0, int step, GET get)
{
    const pr_floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    pr_floatx4 bias[C], bias_up[C];
    pr_uintx4 res[4][C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int n = n0 + step * c;
        bias[c] = o.bias && n < o.N ? load_bias<WHOLE>(o, n) : zero;
        bias_up[c] = ACT == SPEC_ACT_SWIGLU && o.bias && n < o.N ? load_bias<WHOLE>(o, o.N + n) : zero;
    }
    auto ask = [&](int r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int m = m0 + stride * r, n = n0 + step * c;
            res[r & 3][c] = o.residual && m < M && n < o.N ? load_residual<WHOLE>(o, m, n) : (pr_uintx4){0, 0, 0, 0};
        }
    };
#pragma unroll
    for (int r = 0; r < (R < 3 ? R : 3); ++r) ask(r);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r + 3 < R) ask(r + 3);
        const int m = m0 + stride * r;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int n = n0 + step * c;
            const Four f = get(r, c);
            pr_floatx4 v = f.v + bias[c];
            const pr_floatx4 up = f.up + bias_up[c];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = activate<ACT>(v[i]) * (ACT == SPEC_ACT_SWIGLU ? up[i] : 1.f);
            if (o.residual) v += residual_of<WHOLE>(o, res[r & 3][c]);     // (-0 + 0 would be 0)
            if (m < M && n < o.N) store<WHOLE>(o, m, n, v);
        }
    }
}
template <bool WHOLE, bool GATED, int R, int C, typename GET>
__device__ __forceinline__ void finish_for(const Out& o, int m0, int stride, int M, int n0, int step, GET get)
{
    if (GATED) return finish_as<SPEC_ACT_SWIGLU, WHOLE, R, C>(o, m0, stride, M, n0, step, get);
    switch (o.act) {   // (the launch's)
    case SPEC_ACT_RELU: return finish_as<SPEC_ACT_RELU, WHOLE, R, C>(o, m0, stride, M, n0, step, get);
    case SPEC_ACT_GELU: return finish_as<SPEC_ACT_GELU, WHOLE, R, C>(o, m0, stride, M, n0, step, get);
    case SPEC_ACT_SILU: return finish_as<SPEC_ACT_SILU, WHOLE, R, C>(o, m0, stride, M, n0, step, get);
    default: return finish_as<SPEC_ACT_NONE, WHOLE, R, C>(o, m0, stride, M, n0, step, get);
    }
}
template <bool GATED, int R, int C, typename GET>
__device__ __forceinline__ void finish(const Out& o, int m0, int stride, int M, int n0, int step, GET get)
{
    if (o.whole) finish_for<true, GATED, R, C>(o, m0, stride, M, n0, step, get);
    else finish_for<false, GATED, R, C>(o, m0, stride, M, n0, step, get);
}

// The 16 RT x 16 CT block of products that a wavefront holds, from row m0 and column tile j0 of W on
template <bool GATED, int RT, int CT>
__device__ __forceinline__ void finish_block(const Out& o, const pr_floatx4 (&acc)[RT][CT], int m0, int j0, int M)
{
    constexpr int S = GATED ? 2 : 1;   // column tiles of W for one of y
    const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    finish<GATED, RT, CT / S>(o, m0 + r16, 16, M, j0 / S * 16 + 4 * g, 16, [&](int r, int c) { return Four{acc[r][S * c], acc[r][S * c + S - 1]}; });
}

__device__ __forceinline__ pr_floatx4 mfma(pr_bf16x8 w, pr_bf16x8 x, pr_floatx4 d) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, d, 0, 0, 0); }

constexpr int TILE = 1024;   // bytes of a 16 x 32 tile of W
constexpr int PANEL = 8;     // row blocks of a panel
constexpr int MAX_COLS = 1 << 23;
constexpr size_t MOST_PARTS = (size_t)1 << 25;   // floats of a workspace that is asked for: where parts pay, they are few

// ---- many rows: the matrix cores ----------------------------------------------------------------------------------------
//
// WR x WC wavefronts take 16 WR RT rows by 16 WC CT columns.  A stage is 64 columns of K: SX stages of X and SW of W are under way or in use, fetched
// straight into LDS.  W's tiles are in operand order.  X's rows are 128 bytes, the 16-byte pieces of row n in the order piece ^ (n & 7):
// eight lanes fetch a whole line of memory, and the eight lanes of an LDS cycle read eight different groups of banks.
//
// A stage is 2 RT steps of CT products (32 columns of K by RT row tiles, twice).  Nothing is waited for in a row: X's operand is read from LDS
// AHEAD steps before its products, W's half a stage before, and the requests for later stages go out one by one between the products -- all at
// once they keep the wavefront from its products for as long as the fetch of a stage takes (2048 x 22016 x 4096, gate and up: 343 us, between the
// products 280).  The wavefronts meet AHEAD steps before a stage's end: there the stage is in registers, its place is free, and the next one has
// to be there.
//
// What bounds it: large products the power of the card -- 4096 x 4096 x 8192 runs at 1.47 PFLOP/s, with zeros for operands at 1.92 -- others the
// tiles that do not fill the compute units' last turn, and some 8 us of launch, first fetch and epilogue: 1333 x 4104 x 2080 in 231 tiles 28.9 us.
template <bool GATED, int WR, int WC, int RT, int CT, int SX, int SW, int AHEAD>
__global__ void __launch_bounds__(64 * WR * WC, 2) tiled_kernel(const uint16_t* __restrict__ x, const uint8_t* __restrict__ w, int64_t ld_x, int M, int K, int n_tiles, int row_blocks,
                                                      int col_blocks, int splits, int per_split, Out out, float* __restrict__ partial)
{
    constexpr int W = WR * WC, BR = WR * RT, BC = WC * CT;     // row and column tiles of the workgroup
    constexpr int KX = 2 * BR, KW = 2 * BC, UX = KX / W, UW = KW / W;   // KiB of a stage, requests of a wavefront
    constexpr int STEPS = 2 * RT;
    static_assert(KX % W == 0 && KW % W == 0, "every wavefront has as many requests");
    static_assert(SX * KX + SW * KW <= 160, "LDS");
    static_assert(AHEAD <= RT, "reads");
    __shared__ __attribute__((aligned(16))) char lds[(SX * KX + SW * KW) * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int wr = wave / WC, wc = wave % WC;
    // An XCD takes neighbouring tiles: panels of PANEL row blocks, column block by column block, so that the 32 compute units of an XCD work on some
    // 8 by 4 tiles and its L2 has each operand once (8192 x 8192 x 8192: 832 us; all row blocks of one column block at a time: 901)
    const int tiles = row_blocks * col_blocks, total = tiles * splits, xcd = blockIdx.x & 7, each = total >> 3, more = total & 7;
    const int id = xcd * each + min(xcd, more) + (blockIdx.x >> 3), split = id / tiles, tile = id - split * tiles;
    const int panel = tile / (PANEL * col_blocks), in_panel = tile - panel * PANEL * col_blocks, high = min(PANEL, row_blocks - panel * PANEL);
    const int m0 = (panel * PANEL + in_panel % high) * BR * 16, j0 = in_panel / high * BC;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const int n_kb = K >> 5, stage0 = split * per_split, n_stages = min(((n_kb + 1) >> 1) - stage0, per_split);

    // Request u of X is eight rows, of W half a column tile's stage.  Rows and columns beyond the end are the last ones again (never stored); beyond
    // K the pieces of X are the ones before again.
    uint32_t x_off[UX], w_off[UW];
    const uint32_t piece = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
    for (int u = 0; u < UX; ++u) x_off[u] = (uint32_t)(min(m0 + 8 * (W * u + wave) + (lane >> 3), M - 1) - m0) * (uint32_t)(2 * ld_x) + piece;
#pragma unroll
    for (int u = 0; u < UW; ++u) w_off[u] = (uint32_t)min((W * u + wave) / 2, n_tiles - 1 - j0) * (4 * TILE) + ((W * u + wave) & 1) * TILE + lane * 16;
    const char* const xb = (const char*)(x + (size_t)m0 * ld_x);
    const uint8_t* const wb = w + (size_t)j0 * (4 * TILE);
    const uint32_t back = piece & 64;   // of the last stage where K ends in its middle
    auto request_x = [&](int u, int stage, int slot) {
        stage += stage0;
        const uint32_t off = 2 * stage + 2 > n_kb ? x_off[u] - back : x_off[u];
        q8_fetch_lds(xb + (size_t)stage * 128, off, lds0 + (slot * KX + W * u + wave) * 1024);
    };
    auto request_w = [&](int u, int stage, int slot) {
        stage += stage0;
        q8_fetch_lds(wb + (size_t)(stage >> 1) * n_tiles * (4 * TILE) + (stage & 1) * (2 * TILE), w_off[u],
                     lds0 + (SX * KX + slot * KW + W * u + wave) * 1024);
    };
    pr_floatx4 acc[RT][CT];
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int b = 0; b < CT; ++b) acc[a][b] = (pr_floatx4){0.f, 0.f, 0.f, 0.f};

    // A stage's places are free where the wavefronts meet in it (release s); then X of stage s + SX and W of stage s + SW are requested.  Release -1
    // counts what the places hold at first but for the last ones, which stage 0 requests.
    for (int s = 0; s < SW - 1; ++s) {
#pragma unroll
        for (int u = 0; u < UW; ++u) request_w(u, s, s);
        if (s < SX - 1)
#pragma unroll
            for (int u = 0; u < UX; ++u) request_x(u, s, s);
    }
    q8_wait_fetches<0>();
    q8_barrier();
#pragma unroll
    for (int r = 0; r < UX + UW; ++r) {     // (what would be requested in front of stage 0)
        if (r * STEPS / (UX + UW) >= AHEAD) continue;
        if (r < UX) request_x(r, SX - 1, SX - 1);
        else request_w(r - UX, SW - 1, SW - 1);
    }

    const char* const w_at = lds + SX * KX * 1024 + wc * CT * 2 * TILE + lane * 16;
    const char* const x_at = lds + wr * RT * 2048 + r16 * 128;
    const uint32_t x_piece = ((g ^ (r16 & 7)) * 16);
    pr_bf16x8 wf[2][CT], xf[AHEAD + 1];
    uint32_t x_slot = 0, w_slot = 0;
    auto read_w = [&](int h, int b, uint32_t slot) { wf[h][b] = *reinterpret_cast<const pr_bf16x8*>(w_at + slot * (KW * 1024) + (2 * b + h) * TILE); };
    auto read_x = [&](int t, int to, uint32_t slot) {
        xf[to] = *reinterpret_cast<const pr_bf16x8*>(x_at + slot * (KX * 1024) + (t % RT) * 2048 + (x_piece ^ (t / RT * 64)));
    };
#pragma unroll
    for (int b = 0; b < CT; ++b) read_w(0, b, 0);
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) read_x(t, t, 0);
    // The operand of step t is register t % (AHEAD + 1); as STEPS is a multiple of that, the same ones in every stage.
    // PX, PW: the rest of release s - 1 is requested here, CX, CW: the beginning of release s.  LATER: the requests behind those that the next
    // stage needs.
    static_assert(STEPS % (AHEAD + 1) == 0, "registers");
    const unsigned tail = 2 * (stage0 + n_stages) > n_kb ? 0u : ~0u;   // K ends in the middle of the last stage: what lies behind is taken for zeros
    constexpr int D = SW - SX, LATER = (SX - 2) * (UX + UW) + D * UW;
    static_assert(SX >= 2 && (D == 0 || D == 1), "order of requests");
    auto stage = [&](int s, auto px, auto pw, auto cx, auto cw, auto last) {
        constexpr bool PX = decltype(px)::value, PW = decltype(pw)::value, CX = decltype(cx)::value, CW = decltype(cw)::value, LAST = decltype(last)::value;
        const uint32_t x_next = x_slot == SX - 1 ? 0 : x_slot + 1, w_next = w_slot == SW - 1 ? 0 : w_slot + 1;
        const uint32_t x_prev = x_slot == 0 ? SX - 1 : x_slot - 1, w_prev = w_slot == 0 ? SW - 1 : w_slot - 1;
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            const bool met = t >= STEPS - AHEAD;
            if (t == STEPS - AHEAD && !LAST) {
                q8_wait_lds();
                q8_wait_fetches<PX && PW ? LATER : 0>();
                q8_barrier();
            }
            if (t + AHEAD < STEPS) read_x(t + AHEAD, (t + AHEAD) % (AHEAD + 1), x_slot);
            else if (!LAST) read_x(t + AHEAD - STEPS, (t + AHEAD) % (AHEAD + 1), x_next);
            if (t < RT) {
#pragma unroll
                for (int b = t; b < CT; b += RT) read_w(1, b, w_slot);
            }
            if (met && !LAST) {
#pragma unroll
                for (int b = t - (STEPS - AHEAD); b < CT; b += AHEAD) read_w(0, b, w_next);
            }
            const int i = met ? t - (STEPS - AHEAD) : t + AHEAD;   // steps behind the release
#pragma unroll
            for (int r = 0; r < UX + UW; ++r) {
                if (r * STEPS / (UX + UW) != i) continue;
                if (r < UX && (met ? CX : PX)) request_x(r, met ? s + SX : s - 1 + SX, met ? x_slot : x_prev);
                if (r >= UX && (met ? CW : PW)) request_w(r - UX, met ? s + SW : s - 1 + SW, met ? w_slot : w_prev);
            }
            pr_bf16x8 xo = xf[t % (AHEAD + 1)];
            if (LAST && t >= RT) xo = __builtin_bit_cast(pr_bf16x8, __builtin_bit_cast(pr_uintx4, xo) & tail);
#pragma unroll
            for (int b = 0; b < CT; ++b) acc[t % RT][b] = mfma(wf[t / RT][b], xo, acc[t % RT][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        x_slot = x_next;
        w_slot = w_next;
    };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    int s = 0;
    for (; s + SW < n_stages; ++s) stage(s, yes, yes, yes, yes, no);   // (n_stages > SW)
    if (D) stage(s++, yes, yes, yes, no, no);
    stage(s++, yes, std::bool_constant<D == 0>(), no, no, no);
#pragma unroll
    for (int i = 0; i < SX - 2; ++i) stage(s++, no, no, no, no, no);
    stage(s, no, no, no, no, yes);
    if (partial) {
        const int ld = n_tiles * 16;
        const Out part{partial + (size_t)split * M * ld, nullptr, nullptr, ld, 0, 0, SPEC_DTYPE_FP32, SPEC_ACT_NONE, ld, true};
        finish_block<false, RT, CT>(part, acc, m0 + wr * RT * 16, j0 + wc * CT, M);
    } else {
        finish_block<GATED, RT, CT>(out, acc, m0 + wr * RT * 16, j0 + wc * CT, M);
    }
}

// The parts' sums, in their order, and the epilogue: four columns of y a thread
template <bool GATED>
__global__ void __launch_bounds__(256) join_kernel(const float* __restrict__ partial, int splits, int M, int n_tiles, Out out)
{
    const int groups = (out.N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)M * groups) return;
    const int m = (int)(i / groups), n = (int)(i % groups) * 4, ld = n_tiles * 16;
    const int at = GATED ? (n >> 4) * 32 + (n & 15) : n;   // gate tile, up tile
    const float* p = partial + (size_t)m * ld + at;
    const size_t step = (size_t)M * ld;
    pr_floatx4 v = *reinterpret_cast<const pr_floatx4*>(p), up = v;
    if (GATED) up = *reinterpret_cast<const pr_floatx4*>(p + 16);
    for (int s = 1; s < splits; ++s) {
        v += *reinterpret_cast<const pr_floatx4*>(p + s * step);
        if (GATED) up += *reinterpret_cast<const pr_floatx4*>(p + s * step + 16);
    }
    finish<GATED, 1, 1>(out, m, 0, M, n, 0, [&](int, int) { return Four{v, up}; });
}

// ---- few rows: the stream of W ------------------------------------------------------------------------------------------
//
// A workgroup takes 16 RT rows by 16 NT columns; its wavefronts share out K by 128 columns and add their sums up in LDS.  Both operands go
// straight into registers, the next 128 columns' while this one's products run.  Memory bounds it: 8 x 32000 x 4096 38.5 us, 6.8 TB/s of weights (some
// of which stay in the card's last cache from one call to the next).
template <bool GATED, int RT, int NT, int WAVES>
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
    struct Loaded {
        pr_uintx4 w[NT][4], x[RT][4];
    };
    auto load = [&](Loaded& l, int q) {
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                l.w[b][k] = __builtin_nontemporal_load(
                    reinterpret_cast<const pr_uintx4*>(w + ((size_t)q * n_tiles + min(j0 + b, n_tiles - 1)) * (4 * TILE) + k * TILE + lane * 16));
#pragma unroll
        for (int a = 0; a < RT; ++a)
#pragma unroll
            for (int k = 0; k < 4; ++k) l.x[a][k] = *reinterpret_cast<const pr_uintx4*>(xr[a] + 32 * min(4 * q + k, n_kb - 1));
    };
    auto multiply = [&](const Loaded& l, int q) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned is = 4 * q + k < n_kb ? ~0u : 0u;   // beyond K: zeros
#pragma unroll
            for (int a = 0; a < RT; ++a) {
                const pr_bf16x8 xf = __builtin_bit_cast(pr_bf16x8, l.x[a][k] & is);
#pragma unroll
                for (int b = 0; b < NT; ++b) acc[a][b] = mfma(__builtin_bit_cast(pr_bf16x8, l.w[b][k]), xf, acc[a][b]);
            }
        }
    };
    Loaded even, odd;
    int q = wave;
    if (q < n_groups) {
        load(even, q);
        for (;;) {
            if (q + WAVES >= n_groups) {
                multiply(even, q);
                break;
            }
            load(odd, q + WAVES);
            multiply(even, q);
            q += WAVES;
            if (q + WAVES >= n_groups) {
                multiply(odd, q);
                break;
            }
            load(even, q + WAVES);
            multiply(odd, q);
            q += WAVES;
        }
    }
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) part[wave][a * NT + b][lane] = acc[a][b];
    __syncthreads();
    // the wavefronts take turns at the blocks (gate and up tile together)
    constexpr int STEP = GATED ? 2 : 1;
    for (int i = wave * STEP; i < RT * NT; i += WAVES * STEP) {
        pr_floatx4 v[STEP];
#pragma unroll
        for (int t = 0; t < STEP; ++t) {
            v[t] = part[0][i + t][lane];
            for (int k = 1; k < WAVES; ++k) v[t] += part[k][i + t][lane];
        }
        const int m = m0 + 16 * (i / NT) + r16;
        finish<GATED, 1, 1>(out, m, 0, M, (j0 + i % NT) / STEP * 16 + 4 * g, 0, [&](int, int) { return Four{v[0], v[STEP - 1]}; });
    }
}

struct Call {
    const uint16_t* x;
    const uint8_t* w;
    int64_t ld_x;
    int M, K, n_tiles;
    Out out;
    hipStream_t s;
    float* partial;         // the workspace
    size_t partial_floats;
};

template <bool GATED, int RT, int NT, int WAVES>
void launch_skinny(const Call& c)
{
    hipLaunchKernelGGL((skinny_kernel<GATED, RT, NT, WAVES>), dim3((c.n_tiles + NT - 1) / NT, (c.M + 16 * RT - 1) / (16 * RT)), dim3(64 * WAVES), 0, c.s, c.x,
                       c.w, c.ld_x, c.M, c.K, c.n_tiles, c.out);
}

template <bool GATED, int WR, int WC, int RT, int CT, int SX, int SW, int AHEAD>
void launch_tiled(const Call& c, int splits = 1, int per_split = 0)
{
    constexpr int BR = WR * RT, BC = WC * CT;
    const int row_blocks = (c.M + 16 * BR - 1) / (16 * BR), col_blocks = (c.n_tiles + BC - 1) / BC;
    if (splits == 1) per_split = (c.K + 63) / 64;
    hipLaunchKernelGGL((tiled_kernel<GATED, WR, WC, RT, CT, SX, SW, AHEAD>), dim3(row_blocks * col_blocks * splits), dim3(64 * WR * WC), 0, c.s, c.x, c.w, c.ld_x,
                       c.M, c.K, c.n_tiles, row_blocks, col_blocks, splits, per_split, c.out, splits > 1 ? c.partial : nullptr);
    if (splits > 1) {
        const int64_t threads = (int64_t)c.M * ((c.out.N + 3) / 4);
        hipLaunchKernelGGL(join_kernel<GATED>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, c.s, c.partial, splits, c.M, c.n_tiles, c.out);
    }
}

// Which tile, and among how many workgroups K is shared out.  us: a stage of 64 columns, with a workgroup on a compute unit and (where two fit) with two
// on each; measured over K = 4096 and 8192, 48 to 8192 rows, 1024 to 32000 columns (shorter K is priced by the same figures).  A launch
// takes some 3.5 us besides, one whose parts are joined 2.5 us more and the parts' way to memory and back; none is faster than the weights come from memory.
// Gate and up in 32 rows have two wavefronts instead of four (a stage 0.22).
struct Shape {
    int rows, cols, slots;      // slots: SW, which a part's stages have to exceed
    float us1, us2;             // us2 = 0: one workgroup on a compute unit
};
constexpr Shape SHAPES[] = {{256, 256, 3, 1.4f, 0.f}, {256, 128, 3, 0.8f, 0.f}, {192, 128, 3, 0.66f, 0.f}, {128, 256, 3, 0.8f, 0.f},
                            {128, 128, 3, 0.56f, 0.88f}, {96, 128, 3, 0.48f, 0.70f}, {64, 128, 3, 0.30f, 0.52f}, {64, 64, 4, 0.23f, 0.36f}, {32, 64, 5, 0.19f, 0.30f}};
constexpr int MOST_ROWS = 256, MOST_SPLIT = 1024;   // rows of a tile; workgroups of a launch that shares K out
struct Plan {
    int shape, splits, per_split;   // shape < 0: K is shared out within workgroups
    size_t floats;                  // of the workspace
};
// floats: what the workspace holds
Plan plan(bool gated, int M, int n_tiles, int K, size_t floats)
{
    const int stages = (K + 63) / 64;
    Plan best{-1, 1, stages, 0};
    // One workgroup for all rows of a column tile (or two) where that is at most one on each compute unit and two turns of its wavefronts: 17 to 32 rows of
    // K = 2048 by 512 to 4096 columns 4.7 to 6.6 us, in tiles 6.4 to 7.6; 4096 or 6144 columns of K 1.0 to 1.6 times as long as in tiles
    if (M <= 16 || (M <= 32 && K <= 2048 && n_tiles <= (gated ? 512 : 256))) return best;
    const float stream = (float)((double)n_tiles * 32. * K / 6.2e6);
    float least = FLT_MAX;
    for (int i = 0; i < (int)(sizeof(SHAPES) / sizeof(SHAPES[0])); ++i) {
        const Shape& t = SHAPES[i];
        const int64_t tiles = (int64_t)((M + t.rows - 1) / t.rows) * ((16 * (int64_t)n_tiles + t.cols - 1) / t.cols);
        if (tiles > 0x7fffffff / 8) continue;
        for (int splits = 1; splits <= 8; ++splits) {
            const int per = (stages + splits - 1) / splits;
            const size_t need = splits > 1 ? (size_t)splits * M * n_tiles * 16 : 0;
            if (need > floats || (splits > 1 && tiles * splits > MOST_SPLIT)) break;   // (nor would more of them do)
            if (stages - (splits - 1) * per <= t.slots) continue;
            const int wgs = (int)tiles * splits, at_once = t.us2 ? 512 : 256, whole = wgs / at_once, rest = wgs % at_once;
            const float round = (float)whole * (t.us2 ? t.us2 : t.us1) + (rest == 0 ? 0.f : rest <= 256 ? t.us1 : t.us2);
            const float work = round * per * (gated && t.rows == 32 ? 1.16f : 1.f), join = splits > 1 ? 2.5f + (float)need * 8e-6f / 5.f : 0.f;
            const float us = std::max(work, stream) + 0.1f * work + join;
            if (us < least) {
                least = us;
                best = {i, splits, per, need};
            }
        }
    }
    return best;
}

template <bool GATED>
void launch(const Call& c)
{
    const Plan p = plan(GATED, c.M, c.n_tiles, c.K, c.partial_floats);
    switch (p.shape) {
    case 0: return launch_tiled<GATED, 2, 4, 8, 4, 2, 3, 1>(c, p.splits, p.per_split);
    case 1: return launch_tiled<GATED, 4, 2, 4, 4, 3, 3, 3>(c, p.splits, p.per_split);
    case 2: return launch_tiled<GATED, 4, 2, 3, 4, 3, 3, 2>(c, p.splits, p.per_split);
    case 3: return launch_tiled<GATED, 2, 4, 4, 4, 3, 3, 1>(c, p.splits, p.per_split);
    case 4: return launch_tiled<GATED, 2, 2, 4, 4, 2, 3, 1>(c, p.splits, p.per_split);
    case 5: return launch_tiled<GATED, 2, 2, 3, 4, 2, 3, 2>(c, p.splits, p.per_split);
    case 6: return launch_tiled<GATED, 2, 2, 2, 4, 3, 3, 1>(c, p.splits, p.per_split);
    case 7: return launch_tiled<GATED, 2, 2, 2, 2, 3, 4, 1>(c, p.splits, p.per_split);
    case 8: if constexpr (!GATED) return launch_tiled<GATED, 1, 4, 2, 1, 4, 5, 1>(c, p.splits, p.per_split);
            else return launch_tiled<GATED, 1, 2, 2, 2, 4, 5, 1>(c, p.splits, p.per_split);
    }
    // (one row of 4096 x 4096: 6.8 us, 8.2 with two column tiles and eight wavefronts; 8 rows of 32000 x 4096 42.6 with one tile and four, 39.3 with two)
    if (c.M > 32) launch_skinny<GATED, GATED ? 2 : 4, GATED ? 2 : 1, 8>(c);
    else if (c.M > 16) launch_skinny<GATED, 2, GATED ? 2 : 1, 8>(c);
    else if (c.n_tiles >= 1024) launch_skinny<GATED, 1, 2, 4>(c);
    else launch_skinny<GATED, 1, GATED ? 2 : 1, 8>(c);
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_prompt_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t activation)
{
    if (M <= 0 || N <= 0 || K <= 0 || M > SPEC_PROMPT_MAX_ROWS || N > MAX_COLS || K > SPEC_PROMPT_MAX_LD) return 0;
    return 4 * plan(activation == SPEC_ACT_SWIGLU, M, ((activation == SPEC_ACT_SWIGLU ? 2 * N : N) + 15) / 16, K, MOST_PARTS).floats;
}

extern "C" size_t spec_prompt_gemm_workspace_bytes_up_to(int32_t M, int32_t N, int32_t K, int32_t activation)
{
    size_t most = 0;
    for (int m = 1; m <= std::min(M, MOST_ROWS * MOST_SPLIT / 2); ++m)   // (more rows have too many tiles for a second part)
        most = std::max(most, spec_prompt_gemm_workspace_bytes(m, N, K, activation));
    return most;
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
    if (N > MAX_COLS || K > SPEC_PROMPT_MAX_LD)
        return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: N = %d, K = %d, at most %d and %d", N, K, MAX_COLS, SPEC_PROMPT_MAX_LD);
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
                 Out{y, e.bias, e.residual, ld_y, e.ld_residual, e.residual_dtype, y_dtype, e.activation, N, whole}, (hipStream_t)stream, (float*)workspace, workspace ? std::min(workspace_bytes / 4, MOST_PARTS) : 0};
    if ((int64_t)((M + 15) / 16) * n_tiles > (int64_t)1 << 30 || M > SPEC_PROMPT_MAX_ROWS)
        return fail(SPEC_ERR_SHAPE, "spec_prompt_gemm: %d rows of %d columns are too many", M, N);
    if (swiglu) launch<true>(c);
    else launch<false>(c);
    SPECV_LAUNCH_CHECK("spec_prompt_gemm");
    return SPEC_OK;
}
