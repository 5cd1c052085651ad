// Causal attention over packed sequences.  The score product is S^T = K Q^T and the output O^T = V^T P^T, both by 32x32x16 matrix instructions: a
// lane then has one query row, whose maximum and sum it keeps in registers (the other half of the positions is lane ^ 32's), and the
// registers in which the score product leaves P^T are the ones that the second product takes it from, with the positions of 16 in the order
// 8 (e / 4) + 4 (lane / 32) + e % 4.  V^T comes out of LDS by transposing reads in the same order.
//
// A workgroup takes 32 WAVES query rows of one kv head, a row being one query head of one position: the query heads that share a kv head
// share its tile.  Keys and values pass through LDS in blocks of 64 positions, fetched one block ahead, once for all wavefronts.
#include "prompt.h"

namespace specv {
namespace {

constexpr int BLK = 64;   // positions of a block

struct Args {
    const uint16_t *q, *k, *v;
    uint16_t* out;
    int64_t ld_q, ld_k, ld_v, ld_out;
    const int32_t *q_row0, *k_row0;
    int n_kv_heads, group, batch, q_rows, k_rows;
    float factor;       // |scale| * log2(e), not zero: what is masked is -inf times it
    unsigned sign;      // 0x80008000 where the scale is negative: the queries are negated
};

// The largest of lane and lane ^ 32; their sum
__device__ __forceinline__ float both_max(float v)
{
    const pr_uintx2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v)
{
    const pr_uintx2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

typedef short pr_shortx4 __attribute__((ext_vector_type(4)));

template <int HD, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) attention_kernel(Args A)
{
    constexpr int ROW = 2 * HD, PART = BLK * ROW, KIB = PART / 1024;       // bytes of a row, of a block's keys; requests for them
    constexpr int PIECES = ROW / 16, ROWS = 1024 / ROW;                    // 16-byte pieces of a row, rows of a request
    constexpr int U = KIB / WAVES > 0 ? KIB / WAVES : 1;
    static_assert(KIB % WAVES == 0, "every wavefront has as many requests");
    __shared__ __attribute__((aligned(16))) char lds[4 * PART];            // keys, keys, values, values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r32 = lane & 31, half = lane >> 5;
    const int head = blockIdx.x % A.n_kv_heads;
    const int32_t* k_row0 = A.k_row0 ? A.k_row0 : A.q_row0;
    const PromptUnit unit = prompt_unit(blockIdx.x / A.n_kv_heads, A.batch, [&](int b) {
        const PromptSpan s = prompt_span(A.q_row0, b, A.q_rows);
        return ((s.end - s.begin) * A.group + 32 * WAVES - 1) / (32 * WAVES);
    });
    if (unit.seq < 0) return;
    const PromptSpan qs = prompt_span(A.q_row0, unit.seq, A.q_rows), ks = prompt_span(k_row0, unit.seq, A.k_rows);
    const int n_q = qs.end - qs.begin, n_k = ks.end - ks.begin;
    const int n_rows = n_q * A.group, n_tiles = (n_rows + 32 * WAVES - 1) / (32 * WAVES);
    const int tile0 = (n_tiles - 1 - unit.index) * (32 * WAVES);           // the tiles with the longest way first
    const int row = tile0 + wave * 32 + r32;
    const bool live = row < n_rows;
    const int at = min(row, n_rows - 1) / A.group, sub = min(row, n_rows - 1) - at * A.group;
    const int last = n_k - n_q + at;                                        // the last position that this lane's row sees
    const int last_first = n_k - n_q + tile0 / A.group, last_last = n_k - n_q + (min(tile0 + 32 * WAVES, n_rows) - 1) / A.group;
    const int n_blocks = last_last < 0 ? 0 : last_last / BLK + 1;
    const int n_clear = last_first < 0 ? 0 : (last_first + 1) / BLK;       // blocks that all rows see whole

    pr_bf16x8 qf[HD / 16];
    {
        const uint16_t* src = A.q + (size_t)(qs.begin + at) * A.ld_q + (size_t)(head * A.group + sub) * HD + 8 * half;
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) {
            pr_uintx4 v = *reinterpret_cast<const pr_uintx4*>(src + 16 * s);
            v ^= A.sign;
            qf[s] = __builtin_bit_cast(pr_bf16x8, v);
        }
    }

    // A row of LDS holds the pieces of a row of keys in the order piece ^ key_turn(row), of values piece ^ value_turn(row): neighbouring lanes of a
    // read then find different groups of banks
    auto key_turn = [](int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; };
    auto value_turn = [](int r) { return HD == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const char* const kb = (const char*)(A.k + (size_t)ks.begin * A.ld_k + (size_t)head * HD);
    const char* const vb = (const char*)(A.v + (size_t)ks.begin * A.ld_v + (size_t)head * HD);
    auto fetch = [&](int block) {
        const int p0 = block * BLK;
        const char* kp = kb + (size_t)p0 * A.ld_k * 2;
        const char* vp = vb + (size_t)p0 * A.ld_v * 2;
        const uint32_t to = lds0 + (block & 1) * PART;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = wave * U + u, r = i * ROWS + lane / PIECES, piece = lane % PIECES;
            const uint32_t from = (uint32_t)min(r, n_k - 1 - p0);     // (beyond the end: the last row again)
            q8_fetch_lds(kp, from * (uint32_t)(2 * A.ld_k) + (piece ^ key_turn(r)) * 16, to + i * 1024);
            q8_fetch_lds(vp, from * (uint32_t)(2 * A.ld_v) + (piece ^ value_turn(r)) * 16, to + 2 * PART + i * 1024);
        }
    };

    pr_floatx16 o[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    // where this lane reads keys (rows r32, r32 + 32) and values (rows 4 half + (lane & 15) / 4 + 8 j)
    const int v_row = 4 * half + ((lane & 15) >> 2), v_turn = value_turn(v_row);
    auto step = [&](int block, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const char* kl = lds + (block & 1) * PART + r32 * ROW;
        const char* vl = lds + (2 + (block & 1)) * PART + v_row * ROW + (lane & 1) * 8;
        pr_floatx16 s[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[p][i] = 0.f;
#pragma unroll
            for (int c = 0; c < HD / 16; ++c) {
                const pr_bf16x8 kf = *reinterpret_cast<const pr_bf16x8*>(kl + p * 32 * ROW + ((2 * c + half) ^ key_turn(r32)) * 16);
                s[p] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[c], s[p], 0, 0, 0);
            }
        }
        if (MASKED) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (block * BLK + 32 * p + 8 * (i / 4) + 4 * half + i % 4 > last) s[p][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
        top = fmaxf(both_max(top), m);
        if (__any(top > m)) {
            const float f = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * A.factor);
            l *= f;
#pragma unroll
            for (int d = 0; d < HD / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
            m = top;
        }
        const float shift = (MASKED && m == -INFINITY) ? 0.f : m * A.factor;   // (a row that has seen nothing yet)
        pr_bf16x8 pf[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            pr_uintx4 v;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[k / 2][8 * (k % 2) + e], A.factor, -shift));
                const float b = __builtin_amdgcn_exp2f(fmaf(s[k / 2][8 * (k % 2) + e + 1], A.factor, -shift));
                l += a + b;
                v[e / 2] = pr_pack2(a, b);
            }
            pf[k] = __builtin_bit_cast(pr_bf16x8, v);
        }
        bool odd = false;
        if (MASKED) {   // does the block hold a value that a weight of zero does not take away?
            unsigned any = 0;
            const char* part = lds + (2 + (block & 1)) * PART + lane * 16;
#pragma unroll 2
            for (int i = 0; i < KIB; ++i) {
                const pr_uintx4 v = *reinterpret_cast<const pr_uintx4*>(part + i * 1024);
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7f807f80u) + 0x00800080u;
            }
            odd = __any((any & 0x80008000u) != 0);
        }
        auto values = [&](int d, int k) {   // the operand of dims 32 d .. and positions 16 k ..
            const int piece = ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_turn) * 16;
            union {
                pr_shortx4 h[2];
                pr_uintx4 u;
            } vf;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                vf.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) pr_shortx4*)(vl + (16 * k + 8 * j) * ROW + piece));
            return vf.u;
        };
        if (MASKED && odd) {
            // Infinities and NaN apart: what meets a weight that is not zero ends in the sum, by products with ones in their places
            auto pick = [](pr_uintx4 v, unsigned sign) {    // ones where v is NaN or the infinity of that sign
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned bad = ((v[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u, nan = ((v[e] & 0x007f007fu) + 0x7fff7fffu) & 0x80008000u;
                    const unsigned at = bad & (nan | ~(v[e] ^ sign));
                    v[e] = (at >> 15) * 0x3f80u;
                }
                return v;
            };
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
#pragma unroll 1
                for (unsigned sign = 0; sign < 2; ++sign) {
                    pr_floatx16 t;
#pragma unroll
                    for (int i = 0; i < 16; ++i) t[i] = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        asm volatile("" ::: "memory");   // (one operand after the other: this is the rare way, and registers are few)
                        t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pr_bf16x8, pick(values(d, k), sign * 0x80008000u)), pf[k], t, 0, 0, 0);
                    }
                    const float f = sign ? -INFINITY : INFINITY;
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] += t[i] > 0.f ? f : 0.f;
                }
            }
            // (every wavefront has seen the same block, so all come here)
            q8_wait_lds();
            q8_barrier();
            char* own = lds + (2 + (block & 1)) * PART + threadIdx.x * 16;
#pragma unroll 1
            for (int i = 0; i < PART; i += WAVES * 1024) {
                pr_uintx4 v = *reinterpret_cast<const pr_uintx4*>(own + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] &= ~(((((v[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu);
                *reinterpret_cast<pr_uintx4*>(own + i) = v;
            }
            q8_wait_lds();
            q8_barrier();
        }
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pr_bf16x8, values(d, k)), pf[k], o[d], 0, 0, 0);
    };
    if (n_blocks) fetch(0);
    int block = 0;
    auto turn = [&](auto masked) {
        q8_wait_fetches<0>();
        q8_wait_lds();
        q8_barrier();
        if (block + 1 < n_blocks) fetch(block + 1);
        step(block, masked);
    };
    for (; block < n_clear; ++block) turn(std::false_type());
    for (; block < n_blocks; ++block) turn(std::true_type());
    if (!live) return;
    l = both_sum(l);
    const float inv = last < 0 ? 0.f : 1.f / l;
    uint16_t* dst = A.out + (size_t)(qs.begin + at) * A.ld_out + (size_t)(head * A.group + sub) * HD + 4 * half;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const pr_uintx2 v = {pr_pack2(o[d][i] * inv, o[d][i + 1] * inv), pr_pack2(o[d][i + 2] * inv, o[d][i + 3] * inv)};
            *reinterpret_cast<pr_uintx2*>(dst + 32 * d + 2 * i) = v;
        }
}

template <int HD, int WAVES>
void launch(const Args& a, hipStream_t s)
{
    const int64_t tiles = (int64_t)a.q_rows * a.group / (32 * WAVES) + a.batch;
    hipLaunchKernelGGL((attention_kernel<HD, WAVES>), dim3((unsigned)(tiles * a.n_kv_heads)), dim3(64 * WAVES), 0, s, a);
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_prompt_attention_workspace_bytes(int32_t q_rows, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim)
{
    return 0;
}

extern "C" int spec_prompt_attention(const spec_prompt_attn_args* args, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!args) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: NULL arguments");
    const spec_prompt_attn_args& a = *args;
    if (a.n_q_heads <= 0 || a.n_kv_heads <= 0 || a.n_q_heads % a.n_kv_heads || a.n_q_heads > 65536)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: %d query heads, %d kv heads", a.n_q_heads, a.n_kv_heads);
    if (a.head_dim != 64 && a.head_dim != 128) return fail(SPEC_ERR_SHAPE, "spec_prompt_attention: head_dim %d, not 64 or 128", a.head_dim);
    if (a.batch < 0 || a.batch > SPEC_PROMPT_MAX_SEQS || a.q_rows < 0 || a.k_rows < 0 || a.max_q_len < 0 || a.max_k_len < 0)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: %d sequences (at most %d), %d query rows, %d key rows, lengths up to %d and %d", a.batch,
                    SPEC_PROMPT_MAX_SEQS, a.q_rows, a.k_rows, a.max_q_len, a.max_k_len);
    if (!(fabsf(a.scale) <= 3.402823466e38f)) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: scale %g", (double)a.scale);
    const int64_t dq = (int64_t)a.n_q_heads * a.head_dim, dk = (int64_t)a.n_kv_heads * a.head_dim;
    const struct {
        const char* name;
        int64_t ld, least;
    } lds[] = {{"q", a.ld_q, dq}, {"k", a.ld_k, dk}, {"v", a.ld_v, dk}, {"out", a.ld_out, dq}};
    for (const auto& l : lds)
        if (l.ld < l.least || l.ld % 8 || l.ld > SPEC_PROMPT_MAX_LD)
            return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: rows of %s %lld elements apart (at least %lld, a multiple of 8, at most %d)", l.name,
                        (long long)l.ld, (long long)l.least, SPEC_PROMPT_MAX_LD);
    if (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out | (uintptr_t)workspace) & 15)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: q, k, v, out and the workspace have to be 16-byte aligned");
    if (!a.batch || !a.q_rows) return SPEC_OK;
    if (!a.q || !a.out || !a.q_row0 || (a.k_rows && (!a.k || !a.v))) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: null pointer");
    const int group = a.n_q_heads / a.n_kv_heads;
    if ((int64_t)a.q_rows * group > 0x3fffffff || ((int64_t)a.q_rows * group / 32 + a.batch) * a.n_kv_heads > 0x7fffffff)
        return fail(SPEC_ERR_SHAPE, "spec_prompt_attention: %d query rows are too many", a.q_rows);
    const Args g{(const uint16_t*)a.q, (const uint16_t*)a.k, (const uint16_t*)a.v, (uint16_t*)a.out, a.ld_q, a.ld_k, a.ld_v, a.ld_out, a.q_row0,
                 a.k_row0, a.n_kv_heads, group, a.batch, a.q_rows, a.k_rows, fmaxf(fabsf(a.scale) * 1.44269504088896341f, 0x1p-149f), a.scale < 0.f ? 0x80008000u : 0u};
    hipStream_t s = (hipStream_t)stream;
    if (a.head_dim == 128) launch<128, 4>(g, s);
    else launch<64, 4>(g, s);
    SPECV_LAUNCH_CHECK("attention_kernel");
    return SPEC_OK;
}
