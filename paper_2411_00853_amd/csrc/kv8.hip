// The 8-bit KV cache: keys and values of a window into its pages, and the attention that reads them.
#include "q8.h"

#include <atomic>

namespace specv {
namespace {

constexpr int PAGE = SPEC_KV8_PAGE;

// Bytes of (position, dimension) inside a page's keys and values (the orders are the header's)
template <int HD>
__device__ __forceinline__ int key_byte(int t, int d)
{
    return ((t >> 4) * (HD / 16) + (d >> 4)) * 256 + (t & 15) * 16 + (d & 15);
}
__device__ __forceinline__ int value_byte(int t, int d)
{
    return (d >> 5) * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + ((d >> 4) & 1) * 8 + (t >> 4) * 4 + (t & 3);
}

struct Pages {
    uint8_t* data;
    float* scales;
    const int32_t* table;
    int n_pages, n_kv_heads, batch, blocks;
};

// The rows of sequence b; false where there are none or the tables are not what they have to be
__device__ __forceinline__ bool window_of(const int32_t* row0, int b, int rows, int* r0, int* w)
{
    *r0 = row0[b];
    const int r1 = row0[b + 1];
    *w = r1 - *r0;
    return *r0 >= 0 && r1 <= rows && *w > 0;
}

// The smallest power of two s with amax / s <= 448 (448 = 1.75 * 2^8), at least 2^-126
__device__ __forceinline__ float pow2_scale(float amax)
{
    const unsigned u = __float_as_uint(amax);
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    e = max(e, -126);   // also for a magnitude below the normal numbers
    return __uint_as_float((unsigned)(e + 127) << 23);
}

constexpr int APPEND_TPB = 256;

// A workgroup takes one page of one sequence and kv head: its new positions are rotated into LDS, their magnitude and the page's older
// positions decide the scale, and the bytes are written by their one owner.  It also rotates the queries of its heads and rows.
template <int HD>
__global__ void __launch_bounds__(APPEND_TPB) append_kernel(const uint16_t* __restrict__ qkv, const int32_t* __restrict__ row0,
                                                            const int32_t* __restrict__ kv_len, Pages c, const float2* __restrict__ cos_sin,
                                                            int max_pos, int rows, int group, uint16_t* __restrict__ q_out)
{
    __shared__ float fresh[2][PAGE][HD];
    __shared__ unsigned top[2];
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, hk = c.n_kv_heads, hq = hk * group;
    int r0, w;
    if (!window_of(row0, b, rows, &r0, &w)) return;
    const int n = kv_len[b], ld = (hq + 2 * hk) * HD;
    if (n < 0 || n >= c.blocks * PAGE) {   // no place for any row (the first workgroup of a head says so)
        if (q_out && blockIdx.x == 0)
            for (int i = tid; i < w * group * HD; i += APPEND_TPB)
                q_out[(size_t)(r0 + i / (group * HD)) * hq * HD + h * group * HD + i % (group * HD)] = 0;
        return;
    }
    const int blk = n / PAGE + blockIdx.x, lo = max(blk * PAGE, n), hi = (int)min((long)blk * PAGE + PAGE, (long)n + w);
    if (lo >= hi) return;
    const int page = blk < c.blocks ? c.table[(size_t)b * c.blocks + blk] : -1;
    const int seen = min(hi, cos_sin ? max_pos : hi);   // positions the rotation table has
    if (q_out) {   // a thread a pair of dimensions of a query
        for (int i = tid; i < (hi - lo) * group * (HD / 2); i += APPEND_TPB) {
            const int d = i % (HD / 2), k = i / (HD / 2), head = h * group + k % group, pos = lo + k / group, row = r0 + pos - n;
            const uint16_t* src = qkv + (size_t)row * ld + head * HD + d;
            float a = q8_widen(src[0]), o = q8_widen(src[HD / 2]);
            if (cos_sin) {
                const float2 cs = pos < seen ? cos_sin[(size_t)pos * (HD / 2) + d] : make_float2(0.f, 0.f);
                const float x = a * cs.x - o * cs.y;
                o = o * cs.x + a * cs.y;
                a = x;
            }
            const bool in = pos < seen && blk < c.blocks;
            uint16_t* dst = q_out + ((size_t)row * hq + head) * HD + d;
            dst[0] = in ? q8_round_bf16(a) : 0;
            dst[HD / 2] = in ? q8_round_bf16(o) : 0;
        }
    }
    if (page < 0 || page >= c.n_pages || lo >= seen) return;
    if (tid < 2) top[tid] = 0;
    __syncthreads();
    unsigned mk = 0, mv = 0;
    auto grown = [](unsigned m, float f) {   // the largest finite magnitude
        const unsigned u = __float_as_uint(f) & 0x7fffffffu;
        return u < 0x7f800000u ? max(m, u) : m;
    };
    for (int i = tid; i < (seen - lo) * (HD / 2); i += APPEND_TPB) {
        const int d = i % (HD / 2), pos = lo + i / (HD / 2), t = pos - blk * PAGE;
        const uint16_t* src = qkv + (size_t)(r0 + pos - n) * ld + (hq + h) * HD + d;
        float a = q8_widen(src[0]), o = q8_widen(src[HD / 2]);
        if (cos_sin) {
            const float2 cs = cos_sin[(size_t)pos * (HD / 2) + d];
            const float x = a * cs.x - o * cs.y;
            o = o * cs.x + a * cs.y;
            a = x;
        }
        const float v0 = q8_widen(src[hk * HD]), v1 = q8_widen(src[hk * HD + HD / 2]);
        fresh[0][t][d] = a;
        fresh[0][t][d + HD / 2] = o;
        fresh[1][t][d] = v0;
        fresh[1][t][d + HD / 2] = v1;
        mk = grown(grown(mk, a), o);
        mv = grown(grown(mv, v0), v1);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        mk = max(mk, (unsigned)__shfl_xor((int)mk, d));
        mv = max(mv, (unsigned)__shfl_xor((int)mv, d));
    }
    if ((tid & 63) == 0) {
        atomicMax(&top[0], mk);
        atomicMax(&top[1], mv);
    }
    __syncthreads();
    const int older = max(n - blk * PAGE, 0), first = lo - blk * PAGE, last = seen - blk * PAGE;
    float* sc = c.scales + ((size_t)page * hk + h) * 2;
    uint8_t* bytes = c.data + ((size_t)page * hk + h) * (2 * PAGE * HD);
    float was[2], s[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        const float need = pow2_scale(__uint_as_float(top[kv]));
        was[kv] = sc[kv];
        s[kv] = older ? fmaxf(was[kv], need) : need;
    }
    __syncthreads();   // every thread has read the old scales
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        uint8_t* p = bytes + kv * PAGE * HD;
        const float r = 1.f / s[kv];
        for (int i = tid; i < (last - first) * HD; i += APPEND_TPB) {
            const int t = first + i / HD, d = i % HD;
            const float f = fresh[kv][t][d] * r;
            // beyond 448 lie only an infinity and what is not a number
            const unsigned v = fabsf(f) <= 2.f * Q8_MAX ? q8_pack4(f, 0.f, 0.f, 0.f) : 0x7fu;
            p[kv ? value_byte(t, d) : key_byte<HD>(t, d)] = (uint8_t)v;
        }
        if (older && s[kv] > was[kv]) {
            const float f = was[kv] * r;
            for (int i = tid; i < older * HD; i += APPEND_TPB) {
                const int t = i / HD, d = i % HD, at = kv ? value_byte(t, d) : key_byte<HD>(t, d);
                p[at] = (uint8_t)q8_pack4(q8_unpack(p[at]) * f, 0.f, 0.f, 0.f);
            }
        }
        if (tid == 0) sc[kv] = s[kv];
    }
}

// ---- attention ---------------------------------------------------------------------------------------------------------
//
// A wavefront takes 16 RT query rows of one kv head (the heads that share it, window row by window row) and every NWth page of a
// range.  For a page S^T = K Q^T on bf16 (an e4m3 number is one exactly): the result leaves a lane with four neighbouring
// positions of either half of the page for one query, and that is the order in which O^T = V^T P^T takes P^T, on fp16: the
// values are exact in it too, and the weights keep eleven bits.
//
// The scale of a page's values goes into the exponent: the weight that meets the values is exp2(t - ref) with t = score + log2(vs),
// and the sum of weights takes it times 1/vs.  So there is one running reference, of the products' magnitude, and fp16
// holds weights from 2^15 down to 2^-14 above its small numbers: the reference moves only when a weight would pass 2^15.

constexpr float REF_NONE = -1e30f;
constexpr float REF_SLACK = 15.f, REF_BELOW = 6.f;
constexpr float LOG2_VS_LEAST = -80.f;

struct AttnArgs {
    Pages c;
    const uint16_t* q;
    int64_t ld_q;
    const int32_t* row0;
    const int32_t* kv_len;
    int rows, group, parts, tiles;
    float scale;          // of the scores, times log2(e)
    uint16_t* out;
    float* part_o;        // [rows][heads][parts][HD]
    float2* part_ml;      // [rows][heads][parts] reference, sum of weights
};

__device__ __forceinline__ q8_bf16x8 keys8(unsigned a, unsigned b)
{
    const q8_bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const q8_bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return (q8_bf16x8){x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

__device__ __forceinline__ q8_halfx8 values8(unsigned a, unsigned b)
{
    const q8_halfx2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    const q8_halfx2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    return (q8_halfx8){x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

__device__ __forceinline__ bool has_nan(unsigned x) { return (((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }

// The four positions base .. base + 3 of a word, those beyond `last` zero
__device__ __forceinline__ unsigned upto(unsigned x, int base, int last)
{
    const int keep = last - base + 1;   // bytes
    return keep >= 4 ? x : keep <= 0 ? 0u : x & ((1u << (8 * keep)) - 1u);
}

template <int HD, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) attn8_kernel(const AttnArgs a)
{
    constexpr int KC = HD / 64, DT = HD / 16;
    __shared__ q8_floatx4 merged[NW][DT][64];
    __shared__ float2 ml[NW][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int b = blockIdx.z, h = blockIdx.y / a.tiles, q0 = (blockIdx.y % a.tiles) * (16 * RT), hk = a.c.n_kv_heads;
    int r0, w;
    if (!window_of(a.row0, b, a.rows, &r0, &w)) return;
    const int n_q = w * a.group;
    if (q0 >= n_q) return;
    const int cap = a.c.blocks * PAGE, given = a.kv_len[b], n = min(given, cap);
    const int j_lo = q0 / a.group, j_hi = min(n_q - 1, q0 + 16 * RT - 1) / a.group;
    const int len = given < 0 ? 0 : (int)min((long)n + j_hi + 1, (long)cap), n_blk = (len + PAGE - 1) / PAGE;
    const int per = (n_blk + a.parts - 1) / a.parts, c0 = min(n_blk, (int)blockIdx.x * per), c1 = min(n_blk, c0 + per);

    q8_bf16x8 qf[RT][KC][2];
    int lim[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int qi = q0 + 16 * t + r16, qc = min(qi, n_q - 1), j = qc / a.group;
        lim[t] = qi < n_q ? (int)min((long)n + j, (long)cap) : -1;
        const uint16_t* p = a.q + (size_t)(r0 + j) * a.ld_q + (h * a.group + qc % a.group) * HD;
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            const q8_intx4 x = *reinterpret_cast<const q8_intx4*>(p + 64 * k + 16 * g), y = *reinterpret_cast<const q8_intx4*>(p + 64 * k + 16 * g + 8);
            qf[t][k][0] = __builtin_bit_cast(q8_bf16x8, x);
            qf[t][k][1] = __builtin_bit_cast(q8_bf16x8, y);
        }
    }
    const q8_floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    q8_floatx4 o[RT][DT];
    float ref[RT], sum[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        ref[t] = REF_NONE;
        sum[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[t][d] = zero;
    }
    const int32_t* pages = a.c.table + (size_t)b * a.c.blocks;

    for (int blk = c0 + wave; blk < c1; blk += NW) {
        const int page = pages[blk];
        if (page < 0 || page >= a.c.n_pages) continue;
        const size_t at = (size_t)page * hk + h;
        const uint8_t* kp = a.c.data + at * (2 * PAGE * HD) + lane * 16;
        q8_intx4 kr[2][KC], vr[DT / 2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < KC; ++k) kr[s][k] = *reinterpret_cast<const q8_intx4*>(kp + (s * KC + k) * 1024);
#pragma unroll
        for (int d = 0; d < DT / 2; ++d) vr[d] = *reinterpret_cast<const q8_intx4*>(kp + PAGE * HD + d * 1024);
        const float ks = a.c.scales[at * 2] * a.scale, vs = a.c.scales[at * 2 + 1];
        const float lv = fmaxf(__log2f(vs), LOG2_VS_LEAST), inv = exp2f(-lv);

        q8_floatx4 sc[RT][2];
#pragma unroll
        for (int t = 0; t < RT; ++t) sc[t][0] = sc[t][1] = zero;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const q8_bf16x8 k0 = keys8(kr[s][k][0], kr[s][k][1]), k1 = keys8(kr[s][k][2], kr[s][k][3]);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[t][k][0], sc[t][s], 0, 0, 0);
                    sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[t][k][1], sc[t][s], 0, 0, 0);
                }
            }
        const int first = blk * PAGE;
        const bool masked = first + PAGE - 1 > n + j_lo;
        q8_halfx8 p[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            float x[8], m = -INFINITY;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = fmaf(sc[t][s][i], ks, lv);
                    if (masked) v = first + 16 * s + 4 * g + i <= lim[t] ? v : -INFINITY;
                    x[4 * s + i] = v;
                    m = fmaxf(m, v);
                }
            if (__any(m > ref[t] + REF_SLACK)) {
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                const float now = m > ref[t] + REF_SLACK ? m - REF_BELOW : ref[t], f = exp2f(ref[t] - now);
                ref[t] = now;
                sum[t] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[t][d] *= f;
            }
            float add = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = __builtin_amdgcn_exp2f(x[e] - ref[t]);
                add += v;
                p[t][e] = (_Float16)v;
            }
            sum[t] = fmaf(add, inv, sum[t]);
        }
        bool odd = false;   // a masked place holds what is not a number: zero times it would not be zero
        if (masked) {
            unsigned f = 0;
#pragma unroll
            for (int d = 0; d < DT / 2; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) f |= has_nan((unsigned)vr[d][e]);
            odd = __any(f != 0);
        }
        if (!odd) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const q8_halfx8 v = values8((unsigned)vr[d >> 1][(d & 1) * 2], (unsigned)vr[d >> 1][(d & 1) * 2 + 1]);
#pragma unroll
                for (int t = 0; t < RT; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[t], o[t][d], 0, 0, 0);
            }
        } else {
            // one pass for each last visible position: its rows alone take the result, of values cut off behind it
            for (int last = first; last < first + PAGE; ++last) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const bool mine = min(lim[t], first + PAGE - 1) == last;
                    if (!__any(mine)) continue;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const unsigned lo = upto((unsigned)vr[d >> 1][(d & 1) * 2], first + 4 * g, last);
                        const unsigned hi = upto((unsigned)vr[d >> 1][(d & 1) * 2 + 1], first + 16 + 4 * g, last);
                        const q8_floatx4 r = __builtin_amdgcn_mfma_f32_16x16x32_f16(values8(lo, hi), p[t], zero, 0, 0, 0);
                        if (mine) o[t][d] += r;
                    }
                }
            }
        }
    }

    // The wavefronts' results, 16 query rows at a time
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float l = sum[t];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (t) __syncthreads();
        if (lane < 16) ml[wave][lane] = make_float2(ref[t], l);
#pragma unroll
        for (int d = 0; d < DT; ++d) merged[wave][d][lane] = o[t][d];
        __syncthreads();
        for (int i = threadIdx.x; i < DT * 64; i += 64 * NW) {
            const int d = i >> 6, ln = i & 63, qi = q0 + 16 * t + (ln & 15);
            if (qi >= n_q) continue;
            float m = REF_NONE, den = 0.f;
            for (int k = 0; k < NW; ++k) m = fmaxf(m, ml[k][ln & 15].x);
            q8_floatx4 v = zero;
            for (int k = 0; k < NW; ++k) {
                const float2 x = ml[k][ln & 15];
                const float f = exp2f(x.x - m);
                den = fmaf(x.y, f, den);
                v += merged[k][d][ln] * f;
            }
            const int row = r0 + qi / a.group, head = h * a.group + qi % a.group, dim = 16 * d + 4 * (ln >> 4), hq = hk * a.group;
            const size_t at = (size_t)row * hq + head;
            if (a.parts == 1) {
                const float f = den == 0.f ? 0.f : 1.f / den;
                uint16_t* dst = a.out + at * HD + dim;
                const unsigned x = q8_round_bf16(v[0] * f) | (unsigned)q8_round_bf16(v[1] * f) << 16;
                const unsigned y = q8_round_bf16(v[2] * f) | (unsigned)q8_round_bf16(v[3] * f) << 16;
                *reinterpret_cast<uint2*>(dst) = make_uint2(x, y);
            } else {
                const size_t pt = at * a.parts + blockIdx.x;
                *reinterpret_cast<q8_floatx4*>(a.part_o + pt * HD + dim) = v;
                if (dim == 0) a.part_ml[pt] = make_float2(m, den);
            }
        }
    }
}

// A wavefront joins the parts of one (row, head)
template <int HD>
__global__ void __launch_bounds__(64) join_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, uint16_t* __restrict__ out, int parts,
                                                  const int32_t* __restrict__ row0, int batch, int hq)
{
    const size_t at = blockIdx.x;
    if ((int)(at / hq) >= row0[batch]) return;   // a row of no sequence
    const float2* x = part_ml + at * parts;
    float m = REF_NONE, den = 0.f, v[HD / 64];
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) v[i] = 0.f;
    for (int k = 0; k < parts; ++k) m = fmaxf(m, x[k].x);
    for (int k = 0; k < parts; ++k) {
        const float f = exp2f(x[k].x - m);
        den = fmaf(x[k].y, f, den);
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) v[i] = fmaf(part_o[(at * parts + k) * HD + i * 64 + threadIdx.x], f, v[i]);
    }
    const float f = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) out[at * HD + i * 64 + threadIdx.x] = q8_round_bf16(v[i] * f);
}

constexpr int MAX_PARTS = 64;

int compute_units()
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    int n = known[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int HD, int RT>
void launch_attn(AttnArgs a, int batch, int max_window, int max_len, size_t ws_floats, void* ws, hipStream_t s)
{
    constexpr int NW = 4;
    const int hk = a.c.n_kv_heads, hq = hk * a.group;
    a.tiles = (int)(((int64_t)max_window * a.group + 16 * RT - 1) / (16 * RT));
    const int64_t wgs = (int64_t)batch * hk * a.tiles, pages = (max_len + PAGE - 1) / PAGE;
    const size_t each = (size_t)a.rows * hq * (HD + 2);
    int64_t parts = 2 * (int64_t)compute_units() / wgs;
    parts = std::min(parts, (pages + NW - 1) / NW);
    parts = std::min(parts, (int64_t)std::min<size_t>(MAX_PARTS, ws_floats / each));
    a.parts = (int)std::max<int64_t>(parts, 1);
    if (a.parts > 1) {
        a.part_o = (float*)ws;
        a.part_ml = (float2*)(a.part_o + (size_t)a.rows * hq * a.parts * HD);
    }
    hipLaunchKernelGGL((attn8_kernel<HD, RT, NW>), dim3(a.parts, hk * a.tiles, batch), dim3(64 * NW), 0, s, a);
    if (a.parts > 1)
        hipLaunchKernelGGL((join_kernel<HD>), dim3((unsigned)a.rows * hq), dim3(64), 0, s, a.part_o, a.part_ml, a.out, a.parts, a.row0, batch, hq);
}

int check_cache(const char* name, const spec_kv8_cache* c, int n_q_heads, const int32_t* row0, const int32_t* kv_len, int rows, int max_window)
{
    if (!c) return fail(SPEC_ERR_INVALID_ARG, "%s: no cache", name);
    if (c->batch <= 0 || c->n_pages <= 0 || c->blocks_per_seq <= 0 || c->n_kv_heads <= 0 || n_q_heads <= 0 || rows < 0 || max_window < 0)
        return fail(SPEC_ERR_INVALID_ARG, "%s: batch %d, %d pages, %d blocks, %d kv heads, %d query heads, %d rows, window %d", name, c->batch,
                    c->n_pages, c->blocks_per_seq, c->n_kv_heads, n_q_heads, rows, max_window);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(SPEC_ERR_SHAPE, "%s: head_dim %d, 64 and 128 are supported", name, c->head_dim);
    if (n_q_heads % c->n_kv_heads) return fail(SPEC_ERR_SHAPE, "%s: %d query heads on %d kv heads", name, n_q_heads, c->n_kv_heads);
    if (c->batch > 65535 || c->n_kv_heads > 65535 || c->blocks_per_seq > (1 << 25) || max_window > rows || (int64_t)n_q_heads * c->head_dim > (1 << 20))
        return fail(SPEC_ERR_SHAPE, "%s: batch %d, %d kv heads, %d blocks, %d query heads, window %d of %d rows", name, c->batch, c->n_kv_heads,
                    c->blocks_per_seq, n_q_heads, max_window, rows);
    if (!c->data || !c->scales || !c->table || !row0 || !kv_len) return fail(SPEC_ERR_INVALID_ARG, "%s: null pointer", name);
    if ((uintptr_t)c->data & 15) return fail(SPEC_ERR_INVALID_ARG, "%s: the cache is not 16-byte aligned", name);
    return SPEC_OK;
}

Pages pages_of(const spec_kv8_cache* c)
{
    return {(uint8_t*)c->data, c->scales, c->table, c->n_pages, c->n_kv_heads, c->batch, c->blocks_per_seq};
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" int spec_kv8_append(const spec_kv8_cache* cache, const void* qkv, int32_t n_q_heads, const int32_t* row0, const int32_t* kv_len,
                               int32_t rows, int32_t max_window, const float* cos_sin, int32_t max_pos, void* q_out, void* stream)
{
    if (int rc = check_cache("spec_kv8_append", cache, n_q_heads, row0, kv_len, rows, max_window)) return rc;
    if (!rows || !max_window) return SPEC_OK;
    if (!qkv || (cos_sin && !q_out)) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_append: null pointer");
    if (cos_sin && max_pos <= 0) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_append: a rotation of %d positions", max_pos);
    const dim3 grid((max_window + PAGE - 2) / PAGE + 1, cache->n_kv_heads, cache->batch);
    const int group = n_q_heads / cache->n_kv_heads;
    hipStream_t s = (hipStream_t)stream;
    if (cache->head_dim == 64)
        hipLaunchKernelGGL((append_kernel<64>), grid, dim3(APPEND_TPB), 0, s, (const uint16_t*)qkv, row0, kv_len, pages_of(cache),
                           (const float2*)cos_sin, max_pos, rows, group, (uint16_t*)q_out);
    else
        hipLaunchKernelGGL((append_kernel<128>), grid, dim3(APPEND_TPB), 0, s, (const uint16_t*)qkv, row0, kv_len, pages_of(cache),
                           (const float2*)cos_sin, max_pos, rows, group, (uint16_t*)q_out);
    SPECV_LAUNCH_CHECK("append_kernel");
    return SPEC_OK;
}

extern "C" size_t spec_kv8_workspace_bytes(int32_t rows, int32_t n_q_heads, int32_t head_dim)
{
    if (rows <= 0 || n_q_heads <= 0 || head_dim <= 0) return 0;
    // few rows are split the most; many rows fill the chip by themselves
    const size_t each = (size_t)rows * n_q_heads * (head_dim + 2) * sizeof(float);
    return std::min(each * MAX_PARTS, std::max(each * 2, (size_t)64 << 20));
}

extern "C" int spec_kv8_attention(const spec_kv8_cache* cache, const void* q, int64_t ld_q, int32_t n_q_heads, const int32_t* row0,
                                  const int32_t* kv_len, int32_t rows, int32_t max_window, int32_t max_len, float scale, void* out, void* workspace,
                                  size_t workspace_bytes, void* stream)
{
    if (int rc = check_cache("spec_kv8_attention", cache, n_q_heads, row0, kv_len, rows, max_window)) return rc;
    if (!rows || !max_window) return SPEC_OK;
    if (!q || !out) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_attention: null pointer");
    if (((uintptr_t)q & 15) || (ld_q & 7) || ld_q < (int64_t)n_q_heads * cache->head_dim || ((uintptr_t)out & 15) || ((uintptr_t)workspace & 15))
        return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_attention: q, out and workspace have to be 16-byte aligned, rows of q %lld elements apart hold "
                    "%d heads", (long long)ld_q, n_q_heads);
    if (max_len < 0) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_attention: max_len %d", max_len);
    if (!(scale > -INFINITY && scale < INFINITY)) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_attention: scale %g", (double)scale);
    const int cap = cache->blocks_per_seq * PAGE;
    const int group = n_q_heads / cache->n_kv_heads;
    if ((int64_t)cache->n_kv_heads * (((int64_t)max_window * group + 15) / 16) > 65535 || (int64_t)rows * n_q_heads > 0x7fffffff)
        return fail(SPEC_ERR_SHAPE, "spec_kv8_attention: %d rows of %d heads are too many", rows, n_q_heads);
    AttnArgs a{pages_of(cache), (const uint16_t*)q, ld_q, row0, kv_len, rows, group, 1, 1, scale * 1.4426950408889634f, (uint16_t*)out, nullptr, nullptr};
    const size_t ws = workspace ? workspace_bytes / sizeof(float) : 0;
    const int len = max_len ? std::min(max_len, cap) : cap;
    const int n_q = (int)std::min<int64_t>((int64_t)max_window * group, 1 << 20);
    hipStream_t s = (hipStream_t)stream;
#define SPECV_ATTN(HD)                                                                       \
    if (n_q <= 16) launch_attn<HD, 1>(a, cache->batch, max_window, len, ws, workspace, s);   \
    else if (n_q <= 32) launch_attn<HD, 2>(a, cache->batch, max_window, len, ws, workspace, s); \
    else launch_attn<HD, 4>(a, cache->batch, max_window, len, ws, workspace, s)
    if (cache->head_dim == 64) {
        SPECV_ATTN(64);
    } else {
        SPECV_ATTN(128);
    }
#undef SPECV_ATTN
    SPECV_LAUNCH_CHECK("attn8_kernel");
    return SPEC_OK;
}
