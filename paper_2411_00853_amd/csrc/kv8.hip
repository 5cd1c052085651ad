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

// Eight dimensions and the eight they are rotated with
struct Octets {
    float lo[8], hi[8];
};

__device__ __forceinline__ Octets load_octets(const uint16_t* p, int half)
{
    Octets o;
    q8_load8(p, o.lo);
    q8_load8(p + half, o.hi);
    return o;
}

__device__ __forceinline__ void rotate(Octets& o, const float2* cs)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 c = cs[i];
        const float x = o.lo[i] * c.x - o.hi[i] * c.y;
        o.hi[i] = o.hi[i] * c.x + o.lo[i] * c.y;
        o.lo[i] = x;
    }
}

// Two kinds of workgroups for a sequence and kv head.  The first `pages` take one page each: a thread has sixteen dimensions of a new
// position's key and value in registers, their magnitudes and the page's older positions decide the scale, and the bytes are written by
// their one owner.  The rest rotate the queries of the head, sixteen dimensions a thread.  Bound by latency: a window's rows are read,
// its bytes and rotated queries written, 32 sequences of up to 17 rows, 32 query heads and 8 kv heads of 128 in 5 us, one row in 3.9.
template <int HD>
__global__ void __launch_bounds__(APPEND_TPB) append_kernel(const uint16_t* __restrict__ qkv, const int32_t* __restrict__ row0,
                                                            const int32_t* __restrict__ kv_len, const float2* __restrict__ cos_sin, int pages,
                                                            int max_pos, int rows, int group, uint16_t* __restrict__ q_out, Pages c)
{
    constexpr int OCTETS = HD / 16, AT_ONCE = APPEND_TPB / OCTETS;   // positions of a workgroup: 32 or 64
    static_assert(AT_ONCE >= PAGE, "a page's positions at once");
    __shared__ unsigned top[2][APPEND_TPB / 64];
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, hk = c.n_kv_heads, hq = hk * group, oct = tid % OCTETS, d = oct * 8;
    const int n = kv_len[b], ld = (hq + 2 * hk) * HD;
    int r0, w;
    if (!window_of(row0, b, rows, &r0, &w)) return;
    const int limit = min(c.blocks * PAGE, cos_sin ? max_pos : 0x7fffffff);   // positions there is a place for
    if ((int)blockIdx.x >= pages) {
        const int i = ((int)blockIdx.x - pages) * AT_ONCE + tid / OCTETS, j = i / group, head = h * group + i % group;
        if (j >= w) return;
        Octets o = load_octets(qkv + (size_t)(r0 + j) * ld + head * HD + d, HD / 2);
        const long pos = (long)n + j;
        const bool in = n >= 0 && pos < limit;
        if (cos_sin) rotate(o, cos_sin + (in ? pos : 0) * (HD / 2) + d);
        uint16_t lo[8], hi[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo[e] = in ? q8_round_bf16(o.lo[e]) : 0;
            hi[e] = in ? q8_round_bf16(o.hi[e]) : 0;
        }
        uint16_t* dst = q_out + ((size_t)(r0 + j) * hq + head) * HD + d;
        *reinterpret_cast<q8_intx4*>(dst) = *reinterpret_cast<const q8_intx4*>(lo);
        *reinterpret_cast<q8_intx4*>(dst + HD / 2) = *reinterpret_cast<const q8_intx4*>(hi);
        return;
    }
    if (n < 0 || n >= limit) return;
    const int blk = n / PAGE + blockIdx.x;
    const int lo = max(blk * PAGE, n), hi = (int)min((long)min((long)blk * PAGE + PAGE, (long)n + w), (long)limit);
    if (lo >= hi) return;
    const int page = c.table[(size_t)b * c.blocks + blk];
    if (page < 0 || page >= c.n_pages) return;
    float* sc = c.scales + ((size_t)page * hk + h) * 2;
    uint8_t* bytes = c.data + ((size_t)page * hk + h) * (2 * PAGE * HD);
    const float was[2] = {sc[0], sc[1]};
    const int pos = lo + tid / OCTETS, t = pos - blk * PAGE, older = max(n - blk * PAGE, 0);
    const bool mine = pos < hi;
    Octets x[2];
    unsigned most[2] = {0, 0};
    if (mine) {
        const uint16_t* src = qkv + (size_t)(r0 + pos - n) * ld + (hq + h) * HD + d;
        x[0] = load_octets(src, HD / 2);
        x[1] = load_octets(src + hk * HD, HD / 2);
        if (cos_sin) rotate(x[0], cos_sin + (size_t)pos * (HD / 2) + d);
        auto grown = [](unsigned m, float f) {   // the largest finite magnitude
            const unsigned u = __float_as_uint(f) & 0x7fffffffu;
            return u < 0x7f800000u ? max(m, u) : m;
        };
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int e = 0; e < 8; ++e) most[kv] = grown(grown(most[kv], x[kv].lo[e]), x[kv].hi[e]);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        most[kv] = q8_wave_max(most[kv]);
        if ((tid & 63) == 0) top[kv][tid >> 6] = most[kv];
    }
    __syncthreads();   // also: every thread has the old scales
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        unsigned m = 0;
#pragma unroll
        for (int k = 0; k < APPEND_TPB / 64; ++k) m = max(m, top[kv][k]);
        const float need = pow2_scale(__uint_as_float(m)), s = older ? fmaxf(was[kv], need) : need, r = 1.f / s;
        uint8_t* p = bytes + kv * PAGE * HD;
        if (mine) {
            auto byte = [&](float f) {   // beyond 448 lie only an infinity and what is not a number
                f *= r;
                return fabsf(f) <= 2.f * Q8_MAX ? f : __uint_as_float(0x7fc00000u);
            };
            const Octets& v = x[kv];
            const unsigned a0 = q8_pack4(byte(v.lo[0]), byte(v.lo[1]), byte(v.lo[2]), byte(v.lo[3]));
            const unsigned a1 = q8_pack4(byte(v.lo[4]), byte(v.lo[5]), byte(v.lo[6]), byte(v.lo[7]));
            const unsigned b0 = q8_pack4(byte(v.hi[0]), byte(v.hi[1]), byte(v.hi[2]), byte(v.hi[3]));
            const unsigned b1 = q8_pack4(byte(v.hi[4]), byte(v.hi[5]), byte(v.hi[6]), byte(v.hi[7]));
            if (kv == 0) {
                *reinterpret_cast<uint2*>(p + key_byte<HD>(t, d)) = make_uint2(a0, a1);
                *reinterpret_cast<uint2*>(p + key_byte<HD>(t, d + HD / 2)) = make_uint2(b0, b1);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[value_byte(t, d + e)] = (uint8_t)((e < 4 ? a0 : a1) >> (8 * (e & 3)));
                    p[value_byte(t, d + HD / 2 + e)] = (uint8_t)((e < 4 ? b0 : b1) >> (8 * (e & 3)));
                }
            }
        }
        if (older && s > was[kv]) {
            const float f = was[kv] * r;
            for (int i = tid; i < older * HD; i += APPEND_TPB) {
                const int at = kv ? value_byte(i / HD, i % HD) : key_byte<HD>(i / HD, i % HD);
                p[at] = (uint8_t)q8_pack4(q8_unpack(p[at]) * f, 0.f, 0.f, 0.f);
            }
        }
        if (tid == 0) sc[kv] = s;
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
// and the sum of weights takes it times base/vs, with base the scale of the wavefront's first page.  So there is one running reference, of
// the products' magnitude, and fp16 holds weights from 2^15 down to 2^-14 above its small numbers: the reference moves only when a weight
// would pass 2^15.  Scales further apart than 2^+-40 from base would leave weights out of the sum (2^-126 is the least that an exponential
// gives): from the first such page on a wavefront takes t = score + log2(base) against the reference, sums that, and the factor vs/base
// of the weights that meet the values has a running reference of its own, `lift`.  In either case
//     sum of weights = sum * 2^(ref - log2(base)),   O = o * 2^(ref + lift),   out = o / sum * 2^(lift + log2(base)),
// and results are joined by S = ref - log2(base) and E = lift + log2(base), small numbers that no large score swallows.
//
// Bound by the stream of the cache: 8 sequences of 2048 with 32 kv heads of 128, 136 MB in 23.5 us (5.8 TB/s); 32 of 512 to 16384 with 8, 549 MB
// in 103 us (5.3 TB/s).  So every byte is read once for all query heads and window rows that share it; a page's registers are
// filled again as soon as they are free, the keys' while the values are worked on and the other way round (all of a page asked
// for behind its last use: 37.7 us for the first of the two, with the append, against 29); and what runs meanwhile is little: two conversions
// and four products of 16 rows for each 1 KiB.

constexpr float REF_NONE = -0x1.fffffep127f;   // no score is below it
constexpr float REF_SLACK = 15.f, REF_BELOW = 6.f;
constexpr float LOG2_VS_LEAST = -80.f, LOG2_VS_APART = 40.f;

// A result over some positions: the sum of weights is sum * 2^s, the weighted sum of values o * 2^(s + e)
struct Partial {
    float s, sum, e, unused;
};
// Joined: o = sum of o_k * weight_k, out = o * factor(o) (in two steps: 2^most is no fp32 number for the largest scales)
template <int UNROLL, typename F>
__device__ __forceinline__ void join_references(int n, F part, float* top, float* most, float* den)
{
    *top = REF_NONE;
#pragma unroll UNROLL
    for (int k = 0; k < n; ++k) *top = fmaxf(*top, part(k).s);
    *most = REF_NONE;
    *den = 0.f;
#pragma unroll UNROLL
    for (int k = 0; k < n; ++k) {
        const Partial x = part(k);
        *den = fmaf(x.sum, __builtin_amdgcn_exp2f(x.s - *top), *den);
        *most = x.sum == 0.f ? *most : fmaxf(*most, x.s - *top + x.e);
    }
}
__device__ __forceinline__ float join_weight(const Partial& x, float top, float most) { return x.sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(x.s - top + x.e - most); }
__device__ __forceinline__ uint2 finished(const q8_floatx4& o, float most, float den)
{
    const float up = exp2f(0.5f * most), f = den == 0.f ? 0.f : up / den;
    return make_uint2(q8_round_bf16(o[0] * up * f) | (unsigned)q8_round_bf16(o[1] * up * f) << 16,
                      q8_round_bf16(o[2] * up * f) | (unsigned)q8_round_bf16(o[3] * up * f) << 16);
}

struct AttnArgs {
    Pages c;
    const uint16_t* q;
    int64_t ld_q;
    const int32_t* row0;
    const int32_t* kv_len;
    int rows, group, parts, part_pages, tiles, cus;   // part_pages: of each part but a sequence's last, which takes what is left
    float scale;          // of the scores, times log2(e)
    uint16_t* out;
    float* part_o;        // [rows][heads][parts][HD]
    Partial* part_ml;     // [rows][heads][parts]
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

// 0xff in the bytes that are no numbers
__device__ __forceinline__ unsigned nan_bytes(unsigned x) { return ((((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu; }

template <int HD, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) attn8_kernel(const AttnArgs a)
{
    constexpr int KC = HD / 64, DT = HD / 16;
    __shared__ q8_floatx4 merged[NW][DT][64];
    __shared__ Partial ml[NW][16], joined[16];
    __shared__ float weight[NW][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    // (heads fastest: consecutive workgroups go to different XCDs, and a part that many sequences lack would leave one of them idle)
    const int b = blockIdx.z, hk = a.c.n_kv_heads, h = blockIdx.x % hk, q0 = (blockIdx.x / hk) * (16 * RT);
    // (A compute unit's second workgroup takes another part than its first, earlier parts are the longer ones: 106.5 us against 108.6 for 32
    // sequences of 512 to 16384; all first parts first: 115.)
    const int part = (int)((blockIdx.y + gridDim.x * gridDim.y * (unsigned)b / (unsigned)a.cus) % gridDim.y);
    // Asked for at once: the window, the length, and the numbers of the first pages, which the part decides
    const int c0 = part * a.part_pages, given = a.kv_len[b];
    const int32_t* pages = a.c.table + (size_t)b * a.c.blocks;
    const int first_page = pages[min(c0 + wave + lane * NW, a.c.blocks - 1)];
    int r0, w;
    if (!window_of(a.row0, b, a.rows, &r0, &w)) return;
    const int n_q = w * a.group;
    if (q0 >= n_q) return;
    const int cap = a.c.blocks * PAGE, n = min(given, cap);
    const int j_lo = q0 / a.group, j_hi = min(n_q - 1, q0 + 16 * RT - 1) / a.group;
    const int len = given < 0 ? 0 : (int)min((long)n + j_hi + 1, (long)cap), n_blk = (len + PAGE - 1) / PAGE;
    if (part > 0 && part * a.part_pages >= n_blk) {   // nothing to do: says so
        for (int i = threadIdx.x; i < min(16 * RT, n_q - q0); i += 64 * NW) {
            const int qi = q0 + i;
            a.part_ml[((size_t)(r0 + qi / a.group) * hk * a.group + h * a.group + qi % a.group) * a.parts + part] = {REF_NONE, 0.f, 0.f, 0.f};
        }
        return;
    }
    const int c1 = part == a.parts - 1 ? n_blk : min(n_blk, c0 + a.part_pages);

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
    float ref[RT], sum[RT], lift[RT], base = 0.f;   // base: log2 of the scale that the sums are in, the same for the whole wavefront
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        ref[t] = REF_NONE;
        sum[t] = lift[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[t][d] = zero;
    }
    struct Page {
        q8_intx4 k[2][KC], v[DT / 2];
    };
    auto fetch_k = [&](Page& pg, int page) {
        const uint8_t* kp = a.c.data + ((size_t)page * hk + h) * (2 * PAGE * HD) + lane * 16;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < KC; ++k) pg.k[s][k] = __builtin_nontemporal_load(reinterpret_cast<const q8_intx4*>(kp + (s * KC + k) * 1024));
    };
    auto fetch_v = [&](Page& pg, int page) {
        const uint8_t* vp = a.c.data + ((size_t)page * hk + h) * (2 * PAGE * HD) + PAGE * HD + lane * 16;
#pragma unroll
        for (int d = 0; d < DT / 2; ++d) pg.v[d] = __builtin_nontemporal_load(reinterpret_cast<const q8_intx4*>(vp + d * 1024));
    };
    // Scores of page blk against all rows, weights, and the weighted values; the registers of its keys and values take page `next`
    // as soon as they are free.  (These loads are never branched around, or every wait would be for all of them: behind the last page it
    // is read again.)
    auto take = [&](auto scales_apart, Page& pg, int blk, bool there, float ks, float lv, float inv, int next) {
        constexpr bool APART = decltype(scales_apart)::value;
        const auto& kr = pg.k;
        auto& vr = pg.v;
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
                __builtin_amdgcn_sched_barrier(0);   // all of a page widened at once would not fit the registers
            }
        fetch_k(pg, next);
        const int first = blk * PAGE;
        const bool masked = !there || first + PAGE - 1 > n + j_lo;
        q8_halfx8 p[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            float x[8], m = -INFINITY;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = fmaf(sc[t][s][i], ks, APART ? base : lv);
                    if (masked) v = there && first + 16 * s + 4 * g + i <= lim[t] ? v : -INFINITY;
                    x[4 * s + i] = v;
                    m = fmaxf(m, v);
                }
            float up = 0.f;   // log2 of vs / base in units of 2^lift
            if (APART || __any(m > ref[t] + REF_SLACK)) {
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                const float now = m > ref[t] + REF_SLACK ? m - REF_BELOW : ref[t];
                float f = exp2f(ref[t] - now);
                sum[t] *= f;
                if (APART) {
                    // o stays as the reference moves, and follows the largest product; what has no weight yet has no product either
                    const float was = fmaxf(lift[t] + (ref[t] - now), -1e30f), most = m - now + lv - base;
                    lift[t] = most > was + REF_SLACK ? most - REF_BELOW : was;
                    f = exp2f(was - lift[t]);
                    up = lv - base - lift[t];
                }
                ref[t] = now;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[t][d] *= f;
            }
            float add = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = __builtin_amdgcn_exp2f(x[e] - ref[t]);
                add += v;
                p[t][e] = (_Float16)(APART ? __builtin_amdgcn_exp2f(x[e] - ref[t] + up) : v);   // (a small weight of a large scale counts)
            }
            sum[t] = APART ? sum[t] + add : fmaf(add, inv, sum[t]);
        }
        if (masked) {
            unsigned f = 0;
#pragma unroll
            for (int d = 0; d < DT / 2; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) f |= nan_bytes((unsigned)vr[d][e]);
            // Zero times what is not a number is not zero: where a page with a masked place holds one, ones in its place count against
            // ones for the places a row sees, the rows that see it lose that dimension, and zeros go through the product below.
            if (__any(f != 0)) {
                q8_halfx8 seen[RT];
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int e = 0; e < 8; ++e) seen[t][e] = there && first + 16 * (e >> 2) + 4 * g + (e & 3) <= lim[t] ? (_Float16)1.f : (_Float16)0.f;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const unsigned nl = nan_bytes((unsigned)vr[d >> 1][(d & 1) * 2]), nh = nan_bytes((unsigned)vr[d >> 1][(d & 1) * 2 + 1]);
                    const q8_halfx8 ones = values8(nl & 0x38383838u, nh & 0x38383838u);   // 0x38: 1
                    vr[d >> 1][(d & 1) * 2] &= (int)~nl;
                    vr[d >> 1][(d & 1) * 2 + 1] &= (int)~nh;
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const q8_floatx4 r = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, seen[t], zero, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[t][d][i] = r[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[t][d][i];
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const q8_halfx8 v = values8((unsigned)vr[d >> 1][(d & 1) * 2], (unsigned)vr[d >> 1][(d & 1) * 2 + 1]);
#pragma unroll
            for (int t = 0; t < RT; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[t], o[t][d], 0, 0, 0);
            if (d & 1) __builtin_amdgcn_sched_barrier(0);
        }
        fetch_v(pg, next);
    };
    // This wavefront's next 64 pages, one a lane: their numbers and scales.  A page that is not there is read as page 0 and left out.
    int first_blk = c0 + wave;
    auto batches = [&](auto scales_apart) {
        constexpr bool APART = decltype(scales_apart)::value;
        for (; first_blk < c1; first_blk += 64 * NW) {
            const int blk = first_blk + lane * NW, n_mine = min(64, (c1 - first_blk + NW - 1) / NW);
            int page = first_blk == c0 + wave ? first_page : pages[min(blk, c1 - 1)];
            page = blk < c1 ? page : -1;
            const bool there = page >= 0 && page < a.c.n_pages;
            page = there ? page : 0;
            const float2 s2 = *reinterpret_cast<const float2*>(a.c.scales + ((size_t)page * hk + h) * 2);
            const float ks = s2.x * a.scale, lv = there ? fmaxf(__log2f(s2.y), LOG2_VS_LEAST) : 0.f;
            if (!APART) {
                const unsigned long long held = __ballot(there);
                if (first_blk == c0 + wave && held) base = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lv), __builtin_ctzll(held)));
                if (__any(there && fabsf(lv - base) > LOG2_VS_APART)) return;
            }
            const float inv = there && !APART ? exp2f(base - lv) : 1.f;
            const int last = n_mine - 1;
            auto number = [&](int i) { return __builtin_amdgcn_readlane(page, min(i, last)); };
            auto of = [&](float f, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i)); };
            Page pg;
            fetch_k(pg, number(0));
            fetch_v(pg, number(0));
            for (int i = 0; i <= last; ++i)
                take(scales_apart, pg, first_blk + i * NW, __builtin_amdgcn_readlane((int)there, i), of(ks, i), of(lv, i), of(inv, i), number(i + 1));
        }
    };
    batches(std::false_type());
    batches(std::true_type());   // from the first batch on that has scales apart

    // The wavefronts' results, 16 query rows at a time
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float l = sum[t];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (t) __syncthreads();
        if (lane < 16) ml[wave][lane] = {ref[t] - base, l, lift[t] + base, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) merged[wave][d][lane] = o[t][d];
        __syncthreads();
        // (A thread for each wavefront and row: by every thread for itself, 256 workgroups of 64 positions take 5.2 us, 4.6 this way.)
        if (threadIdx.x < NW * 16) {
            const int k = threadIdx.x >> 4, row = lane & 15;
            float top, most, den;
            join_references<NW>(NW, [&](int i) { return ml[i][row]; }, &top, &most, &den);
            weight[k][row] = join_weight(ml[k][row], top, most);
            if (k == 0) joined[row] = {top, den, most, 0.f};
        }
        __syncthreads();
        for (int i = threadIdx.x; i < DT * 64; i += 64 * NW) {
            const int d = i >> 6, ln = i & 63, qi = q0 + 16 * t + (ln & 15);
            if (qi >= n_q) continue;
            const Partial all = joined[ln & 15];
            q8_floatx4 v = zero;
#pragma unroll
            for (int k = 0; k < NW; ++k) v += merged[k][d][ln] * weight[k][ln & 15];
            const int row = r0 + qi / a.group, head = h * a.group + qi % a.group, dim = 16 * d + 4 * (ln >> 4), hq = hk * a.group;
            const size_t at = (size_t)row * hq + head;
            if (a.parts == 1) {
                *reinterpret_cast<uint2*>(a.out + at * HD + dim) = finished(v, all.e, all.sum);
            } else {
                const size_t pt = at * a.parts + part;
                *reinterpret_cast<q8_floatx4*>(a.part_o + pt * HD + dim) = v;
                if (dim == 0) a.part_ml[pt] = all;
            }
        }
    }
}

constexpr int MAX_PARTS = 64;

// `per` (a power of two) groups of HD/4 threads join the parts of one (row, head): a thread has four dimensions of every per-th part.
// Latency: two rounds of loads, 5 us for 143 rows of 32 heads in two parts.
template <int HD>
__global__ void __launch_bounds__(256) join_kernel(const float* __restrict__ part_o, const Partial* __restrict__ part_ml, int parts, int per,
                                                   size_t items, const int32_t* __restrict__ row0, int batch, int hq, uint16_t* __restrict__ out)
{
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
    __shared__ Partial ml[GROUPS][MAX_PARTS];
    __shared__ q8_floatx4 sums[GROUPS][LANES];
    const int tid = threadIdx.x, grp = tid / LANES, dim = (tid % LANES) * 4, item = grp / per, sub = grp % per;
    const size_t at = (size_t)blockIdx.x * (GROUPS / per) + item;
    const bool on = at < items && (int)(at / hq) < row0[batch];   // else a row of no sequence
    if (on)
        for (int k = tid - item * per * LANES; k < parts; k += per * LANES) ml[item][k] = part_ml[at * parts + k];
    __syncthreads();
    q8_floatx4 o = {0.f, 0.f, 0.f, 0.f};
    float top, most = 0.f, den = 0.f;
    if (on) {
        join_references<2>(parts, [&](int k) { return ml[item][k]; }, &top, &most, &den);
#pragma unroll 4
        for (int k = sub; k < parts; k += per) {
            const Partial x = ml[item][k];
            const q8_floatx4 v = *reinterpret_cast<const q8_floatx4*>(part_o + (at * parts + k) * HD + dim);
            o += x.sum == 0.f ? (q8_floatx4){0.f, 0.f, 0.f, 0.f} : v * join_weight(x, top, most);   // a part without a position has written nothing else
        }
    }
    sums[grp][tid % LANES] = o;
    __syncthreads();
    if (!on || sub) return;
    for (int i = 1; i < per; ++i) o += sums[grp + i][tid % LANES];
    *reinterpret_cast<uint2*>(out + at * HD + dim) = finished(o, most, den);
}

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

template <int HD, int RT, int NW>
void launch_attn(AttnArgs a, int batch, int max_window, int max_len, size_t ws_floats, void* ws, hipStream_t s)
{
    const int hk = a.c.n_kv_heads, hq = hk * a.group, cus = compute_units();
    a.tiles = (int)(((int64_t)max_window * a.group + 16 * RT - 1) / (16 * RT));
    const int64_t wgs = (int64_t)batch * hk * a.tiles, pages = (max_len + PAGE - 1) / PAGE;
    const size_t each = (size_t)a.rows * hq * (HD + 4);
    // Parts of a sequence are workgroups of their own, joined by a second kernel (3 us): where there are fewer workgroups than compute units,
    // down to two pages a wavefront -- one sequence of 30000, 8 kv heads: 132 us in one part, 20 in 32; of 2048, 32 heads: 13.6 in one, 10.6
    // in four; of 1024, 8 heads of 64: 6.7 in one, 8.4 in two -- and where sequences may differ by much (32 of 512 to 16384: 106 us in two
    // parts, 107 to 115 in one, 115 in four).
    int64_t parts = (pages + 128) / 256;
    if (wgs < cus && pages * HD > 32 * 128) parts = std::max(parts, std::min((cus + wgs - 1) / wgs, pages / (2 * NW)));
    parts = std::min(parts, (int64_t)std::min<size_t>(MAX_PARTS, ws_floats / each));
    a.parts = (int)std::max<int64_t>(parts, 1);
    a.part_pages = (int)std::max<int64_t>((pages + a.parts - 1) / a.parts, 1);
    if (a.parts > 1) {
        a.part_o = (float*)ws;
        a.part_ml = (Partial*)(a.part_o + (size_t)a.rows * hq * a.parts * HD);
    }
    hipLaunchKernelGGL((attn8_kernel<HD, RT, NW>), dim3(hk * a.tiles, a.parts, batch), dim3(64 * NW), 0, s, a);
    if (a.parts > 1) {
        const int groups = 256 / (HD / 4);
        int per = 1;
        while (per < a.parts && per < groups) per *= 2;
        const size_t items = (size_t)a.rows * hq;
        hipLaunchKernelGGL((join_kernel<HD>), dim3((unsigned)((items * per + groups - 1) / groups)), dim3(256), 0, s, a.part_o, a.part_ml, a.parts, per,
                           items, a.row0, batch, hq, a.out);
    }
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
    const int group = n_q_heads / cache->n_kv_heads, pages = (int)(((int64_t)max_window + PAGE - 2) / PAGE) + 1;
    const int at_once = APPEND_TPB / (cache->head_dim / 16);
    const int64_t queries = q_out ? ((int64_t)max_window * group + at_once - 1) / at_once : 0;
    if (queries + pages > 0x7fffffff) return fail(SPEC_ERR_SHAPE, "spec_kv8_append: a window of %d rows", max_window);
    if (((uintptr_t)q_out | (uintptr_t)qkv) & 15) return fail(SPEC_ERR_INVALID_ARG, "spec_kv8_append: qkv and q_out have to be 16-byte aligned");
    const dim3 grid((unsigned)(pages + queries), cache->n_kv_heads, cache->batch);
    hipStream_t s = (hipStream_t)stream;
    if (cache->head_dim == 64)
        hipLaunchKernelGGL((append_kernel<64>), grid, dim3(APPEND_TPB), 0, s, (const uint16_t*)qkv, row0, kv_len, (const float2*)cos_sin,
                           pages, max_pos, rows, group, (uint16_t*)q_out, pages_of(cache));
    else
        hipLaunchKernelGGL((append_kernel<128>), grid, dim3(APPEND_TPB), 0, s, (const uint16_t*)qkv, row0, kv_len, (const float2*)cos_sin,
                           pages, max_pos, rows, group, (uint16_t*)q_out, pages_of(cache));
    SPECV_LAUNCH_CHECK("append_kernel");
    return SPEC_OK;
}

extern "C" size_t spec_kv8_workspace_bytes(int32_t rows, int32_t n_q_heads, int32_t head_dim)
{
    if (rows <= 0 || n_q_heads <= 0 || head_dim <= 0) return 0;
    // few rows are split the most; many rows fill the chip by themselves
    const size_t each = (size_t)rows * n_q_heads * (head_dim + 4) * sizeof(float);
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
    if ((int64_t)cache->n_kv_heads * (((int64_t)max_window * group + 15) / 16) > 0x7fffffff || (int64_t)rows * n_q_heads > 0x7fffffff)
        return fail(SPEC_ERR_SHAPE, "spec_kv8_attention: %d rows of %d heads are too many", rows, n_q_heads);
    AttnArgs a{pages_of(cache), (const uint16_t*)q, ld_q, row0, kv_len, rows, group, 1, 1, 1, compute_units(), scale * 1.4426950408889634f, (uint16_t*)out, nullptr, nullptr};
    const size_t ws = workspace ? workspace_bytes / sizeof(float) : 0;
    const int len = max_len ? std::min(max_len, cap) : cap;
    const int64_t n_q = (int64_t)max_window * group;
    hipStream_t s = (hipStream_t)stream;
    // Two tiles of 16 query rows a workgroup, which share each page's loads and conversions, once there are workgroups enough without: 32
    // sequences of 512 to 16384 with up to 32 rows per kv head take 107 us, 157 with one tile; 8 of 4096 with 64 rows 25.7 and 23.5.
    // (Four tiles leave one wavefront on a SIMD: 195 and 30.3.)
    const bool two = n_q > 16 && (int64_t)cache->batch * cache->n_kv_heads * ((n_q + 15) / 16) > compute_units();
    if (cache->head_dim == 64) {
        if (two) launch_attn<64, 2, 8>(a, cache->batch, max_window, len, ws, workspace, s);
        else launch_attn<64, 1, 8>(a, cache->batch, max_window, len, ws, workspace, s);
    } else {
        if (two) launch_attn<128, 2, 8>(a, cache->batch, max_window, len, ws, workspace, s);
        else launch_attn<128, 1, 8>(a, cache->batch, max_window, len, ws, workspace, s);
    }
    SPECV_LAUNCH_CHECK("attn8_kernel");
    return SPEC_OK;
}
