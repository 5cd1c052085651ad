// Draws from filtered distributions: temperature, top-k, top-p, min-p, and one given random number per row.
//
// A token's mass is a whole number, so sums over any set are exact in whatever order they are taken.  Tokens are ranked by
// falling logit and rising id; what top-k and top-p keep is a prefix of that order, i.e. everything up to a cut (key, id).
#include "q8.h"

namespace specv {
namespace {

typedef unsigned long long u64;

constexpr int TPB = 1024, WAVES = TPB / 64;
constexpr float MASS_ONE = 0x1p44f;

// Ascending with the logit; -0 and 0 are one value
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

struct Sums {
    u64 a, b;
};

__device__ __forceinline__ Sums block_sums(u64 a, u64 b, Sums* lds)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = {a, b};
    __syncthreads();
    Sums s = lds[0];
    for (int w = 1; w < WAVES; ++w) {
        s.a += lds[w].a;
        s.b += lds[w].b;
    }
    return s;
}

struct Cut {
    unsigned key;   // tokens above it are in, those at it up to id
    int id;
};

// A row of logits, read again by every pass
template <typename T>
struct Row {
    const T* x;
    int vocab;
    float top, t;
    bool greedy;
    u64 least;   // smallest mass kept (min-p), at least 1

    __device__ __forceinline__ float logit(int i) const { return q8_widen(x[i]); }
    __device__ __forceinline__ u64 mass(float l) const
    {
        if (greedy) return l == top ? (u64)MASS_ONE : 0;
        return l > -INFINITY ? (u64)(expf((l - top) / t) * MASS_ONE) : 0;
    }
    __device__ __forceinline__ static bool in(const Cut& c, unsigned key, int i) { return key > c.key || (key == c.key && i <= c.id); }
    // number and mass of the tokens within `c`, of key `from` or more, at least `w_min` heavy, with an id of at most `last`
    __device__ Sums sums(const Cut& c, unsigned from, u64 w_min, int last, Sums* lds) const
    {
        u64 n = 0, m = 0;
        for (int i = threadIdx.x; i <= last; i += TPB) {
            const float l = logit(i);
            const unsigned k = key_of(l);
            if (k < from || !in(c, k, i)) continue;
            const u64 w = mass(l);
            if (w < w_min) continue;
            ++n;
            m += w;
        }
        return block_sums(n, m, lds);
    }
};

// The shortest prefix of the order that holds `need` tokens (by_mass: that mass), within cut `c`: its last token.
// The caller knows that c holds as much.
template <typename T>
__device__ Cut shortest(const Row<T>& r, Cut c, u64 need, bool by_mass, Sums* lds)
{
    unsigned lo = c.key, hi = 0xffffffffu;   // lo holds enough; hi + 1 does not
    while (lo < hi) {
        const unsigned mid = lo + (hi - lo) / 2 + 1;
        const Sums s = r.sums(c, mid, 1, r.vocab - 1, lds);
        if ((by_mass ? s.b : s.a) >= need) lo = mid;
        else hi = mid - 1;
    }
    const unsigned key = lo;
    u64 above = 0;
    if (key != 0xffffffffu) {
        const Sums s = r.sums(c, key + 1, 1, r.vocab - 1, lds);
        above = by_mass ? s.b : s.a;
    }
    int first = 0, last = key == c.key ? c.id : r.vocab - 1;   // the id of the last of the equal ones that is needed
    while (first < last) {
        const int mid = first + (last - first) / 2;
        u64 n = 0, m = 0;
        for (int i = threadIdx.x; i <= mid; i += TPB) {
            const float l = r.logit(i);
            if (key_of(l) != key) continue;
            const u64 w = r.mass(l);
            n += w > 0;
            m += w;
        }
        const Sums s = block_sums(n, m, lds);
        if (above + (by_mass ? s.b : s.a) >= need) last = mid;
        else first = mid + 1;
    }
    return {key, last};
}

template <typename T>
__global__ void __launch_bounds__(TPB) filter_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ uniforms,
                                                     const float* __restrict__ temperature, const int32_t* __restrict__ top_k,
                                                     const float* __restrict__ top_p, const float* __restrict__ min_p,
                                                     int32_t* __restrict__ tokens, float* __restrict__ logprob, int32_t* __restrict__ n_kept,
                                                     float* __restrict__ out)
{
    __shared__ Sums lds[WAVES];
    const int row = blockIdx.x;
    Row<T> r;
    r.x = logits + (size_t)row * ld;
    r.vocab = vocab;
    // the largest logit, and whether the row holds a NaN or a +inf
    unsigned top = 0;
    u64 bad = 0;
    for (int i = threadIdx.x; i < vocab; i += TPB) {
        const float l = r.logit(i);
        if (!(l < INFINITY)) bad = 1;
        else top = max(top, key_of(l));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
    {
        __shared__ unsigned tops[WAVES];
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        bad = block_sums(bad, 0, lds).a;
        for (int w = 0; w < WAVES; ++w) top = max(top, tops[w]);
    }
    r.top = __uint_as_float(top ^ ((top >> 31) ? 0x80000000u : 0xffffffffu));
    r.t = temperature ? temperature[row] : 1.f;
    r.greedy = !(r.t > 0.f);
    if (bad || !(r.top > -INFINITY)) {
        if (threadIdx.x == 0) {
            tokens[row] = -1;
            if (logprob) logprob[row] = __uint_as_float(0x7fc00000u);
            if (n_kept) n_kept[row] = 0;
        }
        if (out)
            for (int i = threadIdx.x; i < vocab; i += TPB) out[(size_t)row * vocab + i] = -INFINITY;
        return;
    }
    Cut c = {0, vocab - 1};
    const Sums all = r.sums(c, 0, 1, vocab - 1, lds);
    u64 z = all.b;
    const int k = r.greedy ? 1 : top_k ? top_k[row] : 0;
    if (k > 0 && (u64)k < all.a) {
        c = shortest(r, c, (u64)k, false, lds);
        z = r.sums(c, 0, 1, vocab - 1, lds).b;
    }
    const float p = top_p ? top_p[row] : 1.f;
    if (p < 1.f) c = shortest(r, c, max((u64)ceil((double)p * (double)z), (u64)1), true, lds);
    const float mp = min_p ? min_p[row] : 0.f;
    r.least = mp > 0.f ? max((u64)ceil(fmin((double)mp, 1.0) * (double)MASS_ONE), (u64)1) : 1;
    const Sums kept = r.sums(c, 0, r.least, vocab - 1, lds);
    u64 target = (u64)((double)uniforms[row] * (double)kept.b);
    target = min(target, kept.b - 1);
    int first = 0, last = vocab - 1;
    while (first < last) {
        const int mid = first + (last - first) / 2;
        if (r.sums(c, 0, r.least, mid, lds).b > target) last = mid;
        else first = mid + 1;
    }
    if (threadIdx.x == 0) {
        tokens[row] = first;
        if (logprob) logprob[row] = (float)log((double)r.mass(r.logit(first)) / (double)kept.b);
        if (n_kept) n_kept[row] = (int)kept.a;
    }
    if (out)
        for (int i = threadIdx.x; i < vocab; i += TPB) {
            const float l = r.logit(i);
            out[(size_t)row * vocab + i] = Row<T>::in(c, key_of(l), i) && r.mass(l) >= r.least ? l : -INFINITY;
        }
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_filter_workspace_bytes(int32_t rows, int32_t vocab)
{
    (void)rows;
    (void)vocab;
    return 0;
}

extern "C" int spec_filter_sample(const spec_filter_args* a, const spec_filter_out* o, void* workspace, size_t workspace_bytes, void* stream)
{
    (void)workspace_bytes;
    if (!a || !o) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: null pointer");
    if (a->rows < 0 || a->vocab <= 0 || a->ld < a->vocab)
        return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: %d rows of %d logits, %lld elements apart", a->rows, a->vocab, (long long)a->ld);
    if (!q8_dtype(a->dtype)) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: unknown type %d", a->dtype);
    if (a->vocab > SPEC_FILTER_MAX_VOCAB) return fail(SPEC_ERR_SHAPE, "spec_filter_sample: vocabulary %d, at most %d", a->vocab, SPEC_FILTER_MAX_VOCAB);
    if (!a->rows) return SPEC_OK;
    if (!a->logits || !a->uniforms || !o->tokens) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: null pointer");
    if ((uintptr_t)workspace & 15) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: the workspace is not 16-byte aligned");
    const dim3 grid(a->rows);
    hipStream_t s = (hipStream_t)stream;
    if (a->dtype == SPEC_DTYPE_BF16)
        hipLaunchKernelGGL((filter_kernel<uint16_t>), grid, dim3(TPB), 0, s, (const uint16_t*)a->logits, a->ld, a->vocab, a->uniforms, a->temperature,
                           a->top_k, a->top_p, a->min_p, o->tokens, o->logprob, o->n_kept, o->logits_out);
    else
        hipLaunchKernelGGL((filter_kernel<float>), grid, dim3(TPB), 0, s, (const float*)a->logits, a->ld, a->vocab, a->uniforms, a->temperature,
                           a->top_k, a->top_p, a->min_p, o->tokens, o->logprob, o->n_kept, o->logits_out);
    SPECV_LAUNCH_CHECK("filter_kernel");
    return SPEC_OK;
}
