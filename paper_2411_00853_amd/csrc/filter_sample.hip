// Draws from filtered distributions: temperature, top-k, top-p, min-p, and one given random number per row.
//
// A token's mass is a whole number, so sums over any set are exact in whatever order they are taken.  Tokens are ranked by
// falling logit and rising id; what top-k and top-p keep is a prefix of that order, i.e. everything up to a cut (key, id).
//
// Bound by what a workgroup does one thing after another, not by memory (64 rows of 128256 are 33 MB, 7 us).  With top-k few tokens
// matter, and they are known after one pass: the k-th largest of the threads' own largest logits is a bound, what reaches it makes a
// list (some dozen tokens for k = 50 of 32000), and the rest is work on that list: 9.6 us for one row of 32000 with its filtered
// row, 17.5 for 64 rows of 128256 (38 with a histogram over the row).  A vector instruction costs the workgroup sixteen cycles, its sixteen
// wavefronts four times four, so that what is done for each logit is counted in instructions.  A histogram of 4096 bins and the tokens of one of them find a cut in
// longer lists and in whole rows; without top-k the passes over the row are shared out, see below.
#include "q8.h"

namespace specv {
namespace {

typedef unsigned long long u64;

constexpr int TPB = 1024, WAVES = TPB / 64;
constexpr int BINS = 4096;      // of falling logits, over the 31 nats in which a token has mass
constexpr int LIST = 2048;      // tokens that may matter, where that few are known to
constexpr int SMALL = 1024;     // tokens of the bin that a cut falls into
constexpr int SHORT = 256;      // tokens of a list that is put in order at once
constexpr int GROUPS = SPEC_FILTER_MAX_VOCAB / (TPB * 32);   // of 32 logits a thread
constexpr float NATS = 31.f;    // exp(-31) * 2^44 < 1
constexpr float HALF_ONE = 0x1p22f;
constexpr u64 MASS_ONE = 1ull << 44;

// ---- a wavefront's sums by DPP ------------------------------------------------------------------------------------------
enum { DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_SHR1 = 0x111, DPP_SHR2 = 0x112, DPP_SHR4 = 0x114, DPP_SHR8 = 0x118, DPP_MIRROR = 0x140,
       DPP_HALF_MIRROR = 0x141, DPP_BCAST15 = 0x142, DPP_BCAST31 = 0x143 };
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp(unsigned v)   // lanes without a source get 0
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp(u64 v)
{
    return (u64)dpp<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | dpp<CTRL, ROWS>((unsigned)v);
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v)   // inclusive
{
    v += dpp<DPP_SHR1, 0xf>(v);
    v += dpp<DPP_SHR2, 0xf>(v);
    v += dpp<DPP_SHR4, 0xf>(v);
    v += dpp<DPP_SHR8, 0xf>(v);
    v += dpp<DPP_BCAST15, 0xa>(v);
    v += dpp<DPP_BCAST31, 0xc>(v);
    return v;
}
__device__ __forceinline__ unsigned last_lane(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ u64 last_lane(u64 v) { return (u64)last_lane((unsigned)(v >> 32)) << 32 | last_lane((unsigned)v); }
template <typename T>
__device__ __forceinline__ T wave_sum(T v)   // the same for all lanes
{
    return last_lane(wave_scan(v));
}
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    v = max(v, dpp<DPP_XOR1, 0xf>(v));
    v = max(v, dpp<DPP_XOR2, 0xf>(v));
    v = max(v, dpp<DPP_HALF_MIRROR, 0xf>(v));
    v = max(v, dpp<DPP_MIRROR, 0xf>(v));
    v = max(v, dpp<DPP_BCAST15, 0xa>(v));
    v = max(v, dpp<DPP_BCAST31, 0xc>(v));
    return last_lane(v);
}

// What LDS holds for the whole workgroup, as a scalar: a branch on it is one, and what only one side needs is not kept through the other
__device__ __forceinline__ int same_for_all(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ unsigned same_for_all(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }

// ---- what a workgroup knows of its row ----------------------------------------------------------------------------------
// Ascending with the logit; -0 and 0 are one value
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(unsigned key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

struct Cut {        // tokens of a larger key are in, those of this key up to id
    unsigned key;
    int id;
    __device__ __forceinline__ bool has(float l, int i) const
    {
        const unsigned k = key_of(l);
        return k > key || (k == key && i <= id);
    }
};

// Larger orders are ranked before
__device__ __forceinline__ u64 order_of(float l, int id) { return (u64)key_of(l) << 32 | (unsigned)~id; }
__device__ __forceinline__ Cut cut_at(u64 order) { return {(unsigned)(order >> 32), (int)~(unsigned)order}; }
// The values of a list (in LDS, its last eight filled up with zeros) up to an order.  All eight are read before one is looked at: read only
// where they count, each would be waited for (153 tokens: 8.5 us, 3 this way).
__device__ __forceinline__ u64 up_to(const u64* order, const u64* value, int n, u64 mine)
{
    u64 sum = 0;
    for (int j = 0; j < n; j += 8) {
        u64 other[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            other[e] = order[j + e];
            v[e] = value[j + e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e] & (0 - (u64)(other[e] >= mine));
    }
    return sum;
}

struct Sums {
    u64 n, mass;
};

struct Lds {
    u64 hist[BINS];
    float lx[LIST];
    int lid[LIST];
    u64 small[SMALL], value[SMALL];
    unsigned count[TPB];
    float most[GROUPS][TPB];        // of each group of loads of a row that is not kept in registers
    u64 order[SHORT], ranked[SHORT], by_id[SHORT];
    Sums wave[WAVES];
    unsigned tops[WAVES];
    int n_list, n_small, bin;
    unsigned least_key;
    u64 above;
    Cut cut;
};

// Masses of a row.  (l - top) / t is the rounded quotient: r is the rounded 1 / t, and one step of correction behind the product
// with it gives what a division does, at a third of the instructions.
struct Masses {
    float top, t, r, per_nat;   // per_nat: bins of one unit of logit
    // (Were 1 / t infinite, as it is for a t of 2^-128 and less, the top's own quotient would be 0 * inf and no token would have mass.)
    __device__ __forceinline__ void set(float temperature)
    {
        t = temperature > 0.f ? fminf(fmaxf(temperature, 0x1p-126f), 0x1.fffffep127f) : 1.f;
        r = 1.f / t;
        per_nat = fminf((float)BINS / (NATS * t), 0x1.fffffep127f);
    }
    __device__ __forceinline__ u64 operator()(float l) const
    {
        const float d = l - top, q = d * r;
        if (!(q >= -NATS - 1.f)) return 0;   // also -inf
        const float e = expf(fmaf(fmaf(-q, t, d), r, q)) * HALF_ONE;
        return (u64)(unsigned)e << 22 | (unsigned)(__builtin_amdgcn_fractf(e) * HALF_ONE);
    }
    __device__ __forceinline__ int bin(float l) const { return (int)fminf((top - l) * per_nat, (float)(BINS - 1)); }
};

// ---- where tokens come from: registers, memory or the list in LDS ----------------------------------------------------------
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Some {
    T v[N];
};

// A thread's load is N logits (vocab >= N), a wavefront's covers CHUNK consecutive ids; chunk c is wavefront c % WAVES's.  NV loads of a
// thread stay in registers, with NV = 0 every pass reads the row again.
template <typename T, int NV, int PER>
struct Row {
    static constexpr int N = PER, CHUNK = 64 * N;
    const T* x;
    int vocab;
    float v[NV ? NV : 1][N];

    // Load k of this thread.  It is never branched around, or every load would be waited for before the next: where less than a load is left
    // it covers the row's last N logits, and those that are another load's become -inf.
    __device__ __forceinline__ int first_id(int k) const { return min((k * TPB + (int)threadIdx.x) * N, vocab - N); }
    __device__ __forceinline__ Some<T, N> fetch(int k) const { return *reinterpret_cast<const Some<T, N>*>(x + first_id(k)); }
    __device__ __forceinline__ void widen(int k, const Some<T, N>& s, float* to) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), want = (k * TPB + (int)threadIdx.x) * N, i = first_id(k);
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = q8_widen(s.v[e]);
        if ((k * WAVES + wave + 1) * CHUNK > vocab) {
#pragma unroll
            for (int e = 0; e < N; ++e) to[e] = i + e >= want ? to[e] : -INFINITY;
        }
    }
    __device__ __forceinline__ void load()
    {
        Some<T, N> s[NV ? NV : 1];
#pragma unroll
        for (int k = 0; k < NV; ++k) s[k] = fetch(k);
#pragma unroll
        for (int k = 0; k < NV; ++k) widen(k, s[k], v[k]);
    }
    // f(chunk, id of the first, N logits): whole wavefronts.  A logit of -inf may stand for one that is not there.
    template <typename F>
    __device__ __forceinline__ void each_vec(F f) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                f(k * WAVES + wave, first_id(k), v[k]);
                __builtin_amdgcn_sched_barrier(0);   // one load's masses at a time: side by side they do not fit the registers
            }
        } else {
            for (int k = 0; k < loads(); k += AHEAD) group(k, true, f);
        }
    }
    // NV = 0: the row goes by groups of AHEAD loads a thread
    static constexpr int AHEAD = N >= 4 ? 32 / N : 8;
    __device__ __forceinline__ int loads() const { return (vocab + TPB * N - 1) / (TPB * N); }
    // each_vec's f for the group of load k; lanes that do not want it read a place that all of them read, and get -inf
    template <typename F>
    __device__ __forceinline__ void group(int k, bool want, F f) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        Some<T, N> s[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) s[j] = *reinterpret_cast<const Some<T, N>*>(x + (want ? first_id(k + j) : 0));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float l[N];
            widen(k + j, s[j], l);
#pragma unroll
            for (int e = 0; e < N; ++e) l[e] = want ? l[e] : -INFINITY;
            f((k + j) * WAVES + wave, first_id(k + j), l);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const   // f(logit, id)
    {
        each_vec([&](int, int i, const float* l) {
#pragma unroll
            for (int e = 0; e < N; ++e) f(l[e], i + e);
        });
    }
};

struct List {
    const Lds* s;
    int n;
    template <typename F>
    __device__ __forceinline__ void each(F f) const
    {
        for (int i = threadIdx.x; i < n; i += TPB) f(s->lx[i], s->lid[i]);
    }
};

// ---- steps of the whole workgroup -------------------------------------------------------------------------------------------
__device__ __forceinline__ Sums block_sums(u64 n, u64 mass, Lds& s)
{
    n = wave_sum(n);
    mass = wave_sum(mass);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = {n, mass};
    __syncthreads();
    Sums r = s.wave[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        r.n += s.wave[w].n;
        r.mass += s.wave[w].mass;
    }
    return r;
}

// The entry of hist[0 .. n) (n a multiple of TPB) in which the running sum reaches `need`, and the sum before it, to s.bin and s.above
// (the first entry, should none reach it)
__device__ __forceinline__ void crossing(Lds& s, int n, u64 need)
{
    const int per = n / TPB, i0 = threadIdx.x * per, wave = threadIdx.x >> 6;
    u64 mine = 0;
    for (int i = 0; i < per; ++i) mine += s.hist[i0 + i];
    const u64 upto = wave_scan(mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s.wave[wave].n = upto;
    if (threadIdx.x == 0) {
        s.bin = 0;
        s.above = 0;
    }
    __syncthreads();
    u64 before = upto - mine;
    for (int w = 0; w < wave; ++w) before += s.wave[w].n;
    if (before < need && before + mine >= need) {
        int i = i0;
        for (; before + s.hist[i] < need; ++i) before += s.hist[i];
        s.bin = i;
        s.above = before;
    }
    __syncthreads();
}

__device__ __forceinline__ void clear(Lds& s, int n)
{
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += TPB) s.hist[i] = 0;
    if (threadIdx.x == 0) s.n_small = 0;
    __syncthreads();
}

// The shortest prefix that holds `need` (tokens, or mass), by bisection: for a bin of more tokens than SMALL, as many equal logits make
template <typename S>
__device__ __forceinline__ Cut bisect(const S& src, const Masses& m, const Cut c, u64 need, bool by_mass, int vocab, Lds& s)
{
    auto value = [&](float l) {
        const u64 w = m(l);
        return by_mass ? w : (u64)(w > 0);
    };
    auto from = [&](unsigned key) {
        u64 v = 0;
        src.each([&](float l, int i) {
            if (key_of(l) >= key && c.has(l, i)) v += value(l);
        });
        return block_sums(v, 0, s).n;
    };
    unsigned lo = c.key, hi = 0xffffffffu;   // lo holds enough; hi + 1 does not
    while (lo < hi) {
        const unsigned mid = lo + (hi - lo) / 2 + 1;
        if (from(mid) >= need) lo = mid;
        else hi = mid - 1;
    }
    const u64 above = lo == 0xffffffffu ? 0 : from(lo + 1);
    int first = 0, last = lo == c.key ? c.id : vocab - 1;   // the id of the last of the equal ones that is needed
    while (first < last) {
        const int mid = first + (last - first) / 2;
        u64 v = 0;
        src.each([&](float l, int i) {
            if (i <= mid && key_of(l) == lo) v += value(l);
        });
        if (above + block_sums(v, 0, s).n >= need) last = mid;
        else first = mid + 1;
    }
    return {lo, last};
}

// The same for a source that holds all tokens of logit `lowest` and more, where the prefix lies: a histogram of falling logits, and the
// tokens of the bin that it ends in, each against each.  c holds as much as needed and becomes the cut; false: the bin is too full.
template <typename S>
__device__ __forceinline__ bool shortest(const S& src, const Masses& m, Cut& c, u64 need, bool by_mass, float lowest, Lds& s)
{
    clear(s, BINS);
    src.each([&](float l, int i) {
        if (l < lowest || !c.has(l, i)) return;
        const u64 w = m(l);
        if (w) atomicAdd(&s.hist[m.bin(l)], by_mass ? w : 1);
    });
    __syncthreads();
    crossing(s, BINS, need);
    const int bin = s.bin;
    const u64 above = s.above;
    src.each([&](float l, int i) {
        if (l < lowest || m.bin(l) != bin || !c.has(l, i)) return;
        const u64 w = m(l);
        if (!w) return;
        const int at = atomicAdd(&s.n_small, 1);
        if (at >= SMALL) return;
        s.small[at] = order_of(l, i);
        s.value[at] = by_mass ? w : 1;
    });
    __syncthreads();
    const int n = same_for_all(s.n_small);
    if (n > SMALL) return false;
    if (threadIdx.x == 0) s.cut = c;
    if (threadIdx.x < 8 && n + threadIdx.x < SMALL) s.small[n + threadIdx.x] = s.value[n + threadIdx.x] = 0;   // (eight are read at a time)
    __syncthreads();
    if ((int)threadIdx.x < n) {
        const u64 mine = s.small[threadIdx.x], upto = above + up_to(s.small, s.value, n, mine);
        if (upto >= need && upto - s.value[threadIdx.x] < need) s.cut = cut_at(mine);
    }
    __syncthreads();
    c = s.cut;
    return true;
}

struct Params {
    int k;
    float p;
    u64 least;   // smallest mass kept
};

struct Results {
    int32_t* token;
    float* logprob;
    int32_t* n_kept;
    float* out;
};

template <typename S>
__device__ __forceinline__ Sums within(const S& src, const Masses& m, const Cut& c, Lds& s)
{
    u64 n = 0, mass = 0;
    src.each([&](float l, int i) {
        if (!c.has(l, i)) return;
        const u64 w = m(l);
        n += w > 0;
        mass += w;
    });
    return block_sums(n, mass, s);
}

__device__ __forceinline__ u64 share(float p, u64 mass) { return max((u64)ceil((double)fmaxf(p, 0.f) * (double)mass), (u64)1); }

// Top-k (if it cuts) and top-p within a source
template <typename S>
__device__ __forceinline__ bool cuts(const S& src, const Masses& m, const Params& a, Cut& c, int vocab, Lds& s)
{
    if (a.k <= 0 && !(a.p < 1.f)) return true;
    Sums all = within(src, m, c, s);
    if (a.k > 0 && (u64)a.k < all.n) {
        if (!shortest(src, m, c, (u64)a.k, false, -INFINITY, s)) return false;
        if (a.p < 1.f) all = within(src, m, c, s);
    }
    if (a.p < 1.f) {
        // what lies `reach` and more below the top weighs less than the share that is cut off, in all
        const float reach = logf((float)vocab * (float)MASS_ONE / ((1.f - fmaxf(a.p, 0.f)) * (float)all.mass)) + 0.05f;
        return shortest(src, m, c, share(a.p, all.mass), true, m.top - fmaxf(reach, 0.05f) * m.t, s);
    }
    return true;
}

// The row with -inf where `kept` says no
template <typename T, int NV, int N, typename F>
__device__ __forceinline__ void write_row(Row<T, NV, N> r, float* out, F kept)
{
    if (!out) return;
    asm("" : "+s"(r.vocab));   // (places counted anew: kept from the loads until here they would not fit the registers)
    r.each_vec([&](int chunk, int i0, const float* l) {
        const int want = (chunk * 64 + (int)(threadIdx.x & 63)) * N;
        if (want >= r.vocab) return;
        if (want + N <= r.vocab) {
            Some<float, N> a;
#pragma unroll
            for (int e = 0; e < N; ++e) a.v[e] = l[e] > -INFINITY && kept(l[e], i0 + e) ? l[e] : -INFINITY;
            *reinterpret_cast<Some<float, N>*>(out + i0) = a;
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (i0 + e >= want && i0 + e < r.vocab) out[i0 + e] = l[e] > -INFINITY && kept(l[e], i0 + e) ? l[e] : -INFINITY;
    });
}

// The draw: s.hist[0 .. 1024) holds the kept masses by chunk of 64 N ids
template <typename T, int N>
__device__ __forceinline__ void draw_from_chunks(const T* x, int vocab, const Masses& m, const Params& a, const Cut& c, float u, const Sums& kept,
                                                 const Results& o, Lds& s)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 target = min((u64)((double)u * (double)kept.mass), kept.mass - 1);
    crossing(s, 1024, target + 1);
    if (wave == 0) {
        u64 w[N], sum = 0;
        const int i0 = s.bin * 64 * N + lane * N;   // (in the order of the ids, also where a load was moved)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = i0 + e < vocab ? q8_widen(x[i0 + e]) : -INFINITY;
            w[e] = m(l);
            if (w[e] < a.least || !c.has(l, i0 + e)) w[e] = 0;
            sum += w[e];
        }
        const u64 before = s.above + wave_scan(sum) - sum;
        if (before <= target && before + sum > target) {
            int at = 0;   // the first whose running sum exceeds the target
            u64 drawn = 0, upto = before;
            bool done = false;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                upto += w[e];
                if (!done && upto > target) {
                    at = e;
                    drawn = w[e];
                    done = true;
                }
            }
            *o.token = i0 + at;
            if (o.logprob) *o.logprob = (float)log((double)drawn / (double)kept.mass);
            if (o.n_kept) *o.n_kept = (int)kept.n;
        }
    }
}

// The draw among the tokens of a cut, and the results.  `list` holds all of them if `listed`.
template <typename T, int NV, int N>
__device__ __forceinline__ void finish(const Row<T, NV, N>& r, const List& list, bool listed, const Masses& m, const Params& a, const Cut& c, float u, const Results& o,
                                       Lds& s)
{
    constexpr int CHUNK = Row<T, NV, N>::CHUNK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    clear(s, 1024);   // the kept masses by chunk of ids
    u64 n = 0;
    if (listed) {
        list.each([&](float l, int i) {
            if (!c.has(l, i)) return;
            const u64 w = m(l);
            if (w < a.least) return;
            ++n;
            atomicAdd(&s.hist[i / CHUNK], w);
        });
    } else {
        r.each_vec([&](int chunk, int i0, const float* l) {
            unsigned hi = 0, lo = 0;   // of 512 masses at most: no carry out of either half
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const u64 w = m(l[e]);
                if (w < a.least || !c.has(l[e], i0 + e)) continue;
                ++n;
                hi += (unsigned)(w >> 22);
                lo += (unsigned)w & 0x3fffffu;
            }
            hi = wave_sum(hi);
            lo = wave_sum(lo);
            if (lane == 0 && chunk < 1024) s.hist[chunk] = ((u64)hi << 22) + lo;
        });
    }
    __syncthreads();
    const Sums kept = block_sums(n, s.hist[threadIdx.x], s);
    draw_from_chunks<T, N>(r.x, r.vocab, m, a, c, u, kept, o, s);
    write_row(r, o.out, [&](float l, int i) { return c.has(l, i) && m(l) >= a.least; });
}

// Up to SHORT tokens that hold everything kept: each finds its place in the order of the logits and of the ids by looking at all
// others, four threads a token, and everything else is two running sums, for which four wavefronts work, one a SIMD, and the
// rest meet them at the barriers.
template <typename T, int NV, int N>
__device__ __forceinline__ void short_list(const Row<T, NV, N>& r, const Masses& m, const Params& a, float u, int n, const Results& o, Lds& s)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool works = wave < SHORT / 64, on = tid < n;
    u64* scan = s.hist;   // sums of the wavefronts
    auto running = [&](u64 v, int slot) {   // inclusive, over the SHORT threads (one barrier)
        u64 t = 0;
        if (works) {
            t = wave_scan(v);
            if (lane == 63) scan[slot * (SHORT / 64) + wave] = t;
        }
        __syncthreads();
        if (works)
            for (int w = 0; w < wave; ++w) t += scan[slot * (SHORT / 64) + w];
        return t;
    };
    auto total = [&](int slot) {
        u64 t = 0;
        for (int w = 0; w < SHORT / 64; ++w) t += scan[slot * (SHORT / 64) + w];
        return t;
    };
    float l = -INFINITY;
    int id = 0, rank = 0, place = 0;
    u64 mass = 0, mine = 0;
    if (works) {
        if (on) {
            l = s.lx[tid];
            id = s.lid[tid];
            mass = m(l);
            mine = order_of(l, id);
        }
        s.order[tid] = mine;   // (behind the list: 0, which no comparison counts)
    }
    __syncthreads();
    {   // four threads an element
        const u64 its = s.order[tid / 4];
        unsigned found = 0;   // rank, and place in the upper half
        for (int j = tid % 4 * 4; j < n; j += 16) {
            u64 other[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) other[e] = s.order[j + e];
#pragma unroll
            for (int e = 0; e < 4; ++e) found += (other[e] > its) + ((unsigned)((unsigned)other[e] > (unsigned)its) << 16);
        }
        found += dpp<DPP_XOR1, 0xf>(found);
        found += dpp<DPP_XOR2, 0xf>(found);
        if (tid % 4 == 0) s.count[tid / 4] = found;
    }
    __syncthreads();
    if (works) {
        rank = (int)(s.count[tid] & 0xffffu);
        place = (int)(s.count[tid] >> 16);
        if (on) s.ranked[rank] = mass;
        else s.ranked[tid] = 0;
    }
    __syncthreads();
    const bool masses = a.p < 1.f;
    const u64 sorted = works ? s.ranked[tid] : 0;   // of rank tid
    const bool in_k = a.k <= 0 || tid < a.k;
    const u64 upto = running(in_k ? sorted : 0, 0);
    const u64 need = masses ? share(a.p, total(0)) : 0;
    const bool keep = works && in_k && sorted >= a.least && (!masses || upto - sorted < need);
    __syncthreads();
    if (works) {
        s.ranked[tid] = keep ? sorted : 0;
        s.by_id[tid] = 0;
    }
    __syncthreads();
    u64 kept = on ? s.ranked[rank] : 0;
    if (on) s.by_id[place] = kept;
    running(works ? (u64)(kept > 0) : 0, 1);
    const u64 mass_here = works ? s.by_id[tid] : 0, end = running(mass_here, 2), all = total(2);
    const u64 target = min((u64)((double)u * (double)all), all - 1);
    if (works && end - mass_here <= target && end > target) s.bin = tid;   // the place of the token drawn
    __syncthreads();
    if (on && place == s.bin) {
        *o.token = id;
        if (o.logprob) *o.logprob = (float)log((double)mass / (double)all);
        if (o.n_kept) *o.n_kept = (int)total(1);
    }
    if (!o.out) return;
    write_row(r, o.out, [&](float, int) { return false; });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // another wavefront's -inf is not to land on a kept logit
    __syncthreads();
    if (on && kept) o.out[id] = l;
}

// A row with more equal logits than a bin's list takes
template <typename T, int N>
__device__ __forceinline__ void slow_row(const T* x, int vocab, const Masses& m, const Params& a, float u, const Results& o, Lds& s)
{
    const Row<T, 0, N> r = {x, vocab, {}};
    Cut c = {0, vocab - 1};
    Sums all = within(r, m, c, s);
    if (a.k > 0 && (u64)a.k < all.n) {
        c = bisect(r, m, c, (u64)a.k, false, vocab, s);
        all = within(r, m, c, s);
    }
    if (a.p < 1.f) c = bisect(r, m, c, share(a.p, all.mass), true, vocab, s);
    finish(r, List{&s, 0}, false, m, a, c, u, o, s);
}

template <typename T, int NV, int N>
__global__ void __launch_bounds__(TPB) filter_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ uniforms,
                                                     const float* __restrict__ temperature, const int32_t* __restrict__ top_k,
                                                     const float* __restrict__ top_p, const float* __restrict__ min_p,
                                                     int32_t* __restrict__ tokens, float* __restrict__ logprob, int32_t* __restrict__ n_kept,
                                                     float* __restrict__ out)
{
    __shared__ Lds s;
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Row<T, NV, N> r;
    r.x = logits + (size_t)row * ld;
    r.vocab = vocab;
    // The parameters that are there, all asked for before the first is waited for (one that is not is read in a place that is)
    const float t_read = (temperature ? temperature : uniforms)[row], p_read = (top_p ? top_p : uniforms)[row];
    const float mp_read = (min_p ? min_p : uniforms)[row], u = uniforms[row];
    const int k_read = (top_k ? top_k : (const int32_t*)uniforms)[row];
    r.load();
    const float t0 = temperature ? t_read : 1.f, mp = min_p ? mp_read : 0.f;
    Params a;
    a.k = t0 > 0.f ? top_k ? k_read : 0 : 1;
    a.p = top_p ? p_read : 1.f;
    a.least = mp > 0.f ? max((u64)ceil(fmin((double)mp, 1.0) * (double)MASS_ONE), (u64)1) : 1;

    // The largest logit, each thread's own, and whether the row holds a NaN or a +inf: by their bits, of which three are looked at at a time.
    // The largest of them signed is the largest logit that is not negative, or a NaN or +inf; else the smallest unsigned is the largest
    // logit; a negative NaN is the largest unsigned.
    int most_signed = (int)0x80000000;
    unsigned most = 0, least_bits = 0xffffffffu;
    float most_here = -INFINITY;
    auto look = [&](int, int, const float* l) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned b = __float_as_uint(l[e]);
            most_signed = max(most_signed, (int)b);
            most = max(most, b);
            least_bits = min(least_bits, b);
            most_here = fmaxf(most_here, l[e]);
        }
    };
    if constexpr (NV > 0) r.each_vec(look);
    else
        for (int k = 0; k < r.loads(); k += r.AHEAD) {
            r.group(k, true, look);
            s.most[k / r.AHEAD][threadIdx.x] = most_here;
            most_here = -INFINITY;
        }
    const bool bad = most_signed >= 0x7f800000 || most > 0xff800000u;
    const float mine = __uint_as_float(most_signed >= 0 ? (unsigned)most_signed : least_bits);
    {
        const unsigned w = wave_max(__any(bad) ? 0xffffffffu : key_of(mine));
        if (lane == 0) s.tops[wave] = w;
    }
    if (threadIdx.x == 0) {
        s.n_list = 0;
        s.n_small = 0;
        s.bin = 0;
        s.least_key = 0xffffffffu;
    }
    __syncthreads();
    unsigned top = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = max(top, s.tops[w]);
    top = same_for_all(top);
    Masses m;
    m.top = logit_of(top);
    if (top == 0xffffffffu || !(m.top > -INFINITY)) {
        if (threadIdx.x == 0) {
            tokens[row] = -1;
            if (logprob) logprob[row] = __uint_as_float(0x7fc00000u);
            if (n_kept) n_kept[row] = 0;
        }
        if (out)
            for (int i = threadIdx.x; i < vocab; i += TPB) out[(size_t)row * vocab + i] = -INFINITY;
        return;
    }
    m.set(t0);

    Cut c = {0, vocab - 1};
    if (a.k == 1) {   // the first token alone
        int first = 0x7fffffff;
        r.each([&](float l, int i) {
            if (l == m.top) first = min(first, i);
        });
        const unsigned w = wave_max(0x7fffffffu - (unsigned)first);
        __syncthreads();
        if (lane == 0) s.tops[wave] = w;
        __syncthreads();
        unsigned best = 0;
        for (int i = 0; i < WAVES; ++i) best = max(best, s.tops[i]);
        c = {top, (int)(0x7fffffffu - best)};
    }
    const Results o = {tokens + row, logprob ? logprob + row : nullptr, n_kept ? n_kept + row : nullptr, out ? out + (size_t)row * vocab : nullptr};
    if (a.k == 1) {
        if (threadIdx.x == 0) {
            *o.token = c.id;
            if (o.logprob) *o.logprob = 0.f;
            if (o.n_kept) *o.n_kept = 1;
        }
        write_row(r, o.out, [&](float, int i) { return i == c.id; });
        return;
    }
    bool listed = false;
    int n_list = 0;
    if (a.k > 1 && a.k <= TPB) {
        // The k-th largest of the threads' largest logits is at most the k-th largest of all: what is as large makes the list.  (By
        // bins of 31 / 1024 nats, one a thread: the k-th is the smallest in its bin at the latest.)
        s.count[threadIdx.x] = 0;
        __syncthreads();
        const bool some = m(mine) > 0;
        const int bin = min(m.bin(mine) / (BINS / TPB), TPB - 1);
        if (some) atomicAdd(&s.count[bin], 1u);
        __syncthreads();
        unsigned upto = wave_scan(s.count[threadIdx.x]);
        if (lane == 63) s.tops[wave] = upto;
        __syncthreads();
        unsigned before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            before += w < wave ? s.tops[w] : 0u;
            all += s.tops[w];
        }
        upto += before;
        if (upto >= (unsigned)a.k && upto - s.count[threadIdx.x] < (unsigned)a.k) s.bin = threadIdx.x;
        __syncthreads();
        const bool few = all < (unsigned)a.k;   // then everything with mass may be among the first k
        if (some && !few && bin <= s.bin) atomicMin(&s.least_key, key_of(mine));
        __syncthreads();
        const float least = few ? -0x1.fffffep127f : logit_of(s.least_key);
        // Each wavefront lists its own first, in a place that it has in s.hist: no lane waits for a count to come back.  A lane looks at up to 32
        // logits, a bit each, and what it found is read again: a hit or two, where logit by logit every lane would go through the motions
        // of listing for any other lane's (64 rows of 128256: 23.3 us that way).
        constexpr int OWN = BINS / WAVES;
        u64* const own = s.hist + wave * OWN;
        int n_own = 0;
        auto hand_over = [&]() {
            int at = 0;
            if (lane == 0) at = atomicAdd(&s.n_list, n_own);
            at = __builtin_amdgcn_readfirstlane(at);
            for (int i = lane; i < n_own && at + i < LIST; i += 64) {
                s.lx[at + i] = __uint_as_float((unsigned)(own[i] >> 32));
                s.lid[at + i] = (int)own[i];
            }
            n_own = 0;
        };
        unsigned found;
        int at_bit;
        auto look_again = [&](int, int, const float* l) {
#pragma unroll
            for (int e = 0; e < N; ++e) found |= (unsigned)(l[e] >= least) << (at_bit + e);
            at_bit += N;
        };
        auto collect = [&](int k) {
            u64 which;
            while ((which = __ballot(found != 0)) != 0) {
                const int n = __popcll(which), bit = __builtin_ctz(found | 0x80000000u), id = r.first_id(k + bit / N) + bit % N;
                if (n_own + n > OWN) hand_over();
                if (found) {
                    const int at = n_own + __builtin_amdgcn_mbcnt_hi((unsigned)(which >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)which, 0));
                    own[at] = (u64)__float_as_uint(q8_widen(r.x[id])) << 32 | (unsigned)id;
                }
                n_own += n;
                found &= found - 1;
            }
        };
        static_assert(NV * N <= 32, "a bit each");
        if constexpr (NV > 0) {
            found = 0;
            at_bit = 0;
            r.each_vec(look_again);
            collect(0);
        } else {
            // The groups of loads that hold one are few (200 of 4096 for k = 150 of 128256): they are listed, and a thread takes a load
            // of one (64 rows: 17.5 us; 21.4 where each thread reads its own groups again).
            unsigned* const work = reinterpret_cast<unsigned*>(s.small);
            constexpr int WORK = 2 * SMALL;
            const int n_groups = (r.loads() + r.AHEAD - 1) / r.AHEAD;
            int mine = 0, at = 0;
            for (int g = 0; g < n_groups; ++g) mine += __popcll(__ballot(s.most[g][threadIdx.x] >= least));
            if (lane == 0) at = atomicAdd(&s.n_small, mine);
            at = __builtin_amdgcn_readfirstlane(at);
            for (int g = 0; g < n_groups; ++g) {
                const bool on = s.most[g][threadIdx.x] >= least;
                const u64 which = __ballot(on);
                const int to = at + __builtin_amdgcn_mbcnt_hi((unsigned)(which >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)which, 0));
                if (on && to < WORK) work[to] = (unsigned)g * TPB + threadIdx.x;
                at += __popcll(which);
            }
            __syncthreads();
            const int n_work = same_for_all(s.n_small);
            if (n_work <= WORK) {
                for (int i0 = wave * 64; i0 < n_work * r.AHEAD; i0 += TPB) {
                    const int i = i0 + lane, item = i / r.AHEAD;
                    const unsigned it = work[min(item, n_work - 1)];
                    const int want = (((int)(it / TPB) * r.AHEAD + i % r.AHEAD) * TPB + (int)(it % TPB)) * N, id = min(want, vocab - N);
                    const Some<T, N> x = *reinterpret_cast<const Some<T, N>*>(r.x + id);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float l = q8_widen(x.v[e]);
                        const bool on = item < n_work && id + e >= want && l >= least;
                        const u64 which = __ballot(on);
                        if (!which) continue;
                        const int n = __popcll(which);
                        if (n_own + n > OWN) hand_over();
                        if (on)
                            own[n_own + __builtin_amdgcn_mbcnt_hi((unsigned)(which >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)which, 0))] =
                                (u64)__float_as_uint(l) << 32 | (unsigned)(id + e);
                        n_own += n;
                    }
                }
            } else {
                for (int k = 0; k < r.loads(); k += r.AHEAD) {
                    found = 0;
                    at_bit = 0;
                    const bool any = s.most[k / r.AHEAD][threadIdx.x] >= least;
                    if (!__any(any)) continue;
                    r.group(k, any, look_again);
                    collect(k);
                }
            }
        }
        hand_over();
        __syncthreads();
        n_list = same_for_all(s.n_list);
        listed = n_list <= LIST;
        if (!few) c.key = s.least_key;   // no token outside the list is in
    }
    if (listed && n_list <= SHORT) {
        short_list(r, m, a, u, n_list, o, s);
        return;
    }
    // From here on the row is read again: its registers would not be registers if whatever follows held on to them.
    const T* x = r.x;
    asm("" : "+s"(x));   // (or the compiler knows what it would read)
    const List list = {&s, n_list};
    const Row<T, 0, N> again = {x, vocab, {}};
    if (listed ? cuts(list, m, a, c, vocab, s) : cuts(again, m, a, c, vocab, s)) finish(again, list, listed, m, a, c, u, o, s);
    else slow_row<T, N>(x, vocab, m, a, u, o, s);
}

// ---- rows shared out among workgroups -------------------------------------------------------------------------------------
//
// Without top-k nothing says early which tokens matter, and every pass goes over the whole row.  Then each pass is a launch of its own, in
// which a workgroup takes a slice of a row; sums over slices are sums of whole numbers, added up in any order.  A workgroup
// takes slices of whole chunks (64 loads), a wavefront a chunk at a time.
constexpr int PART_TPB = 256, PART_WAVES = PART_TPB / 64, MAX_PARTS = 64;
constexpr int MANY = 2048;      // tokens of the bin that top-p's cut falls into

struct Shared {                 // of a row, in the workspace
    u64 hist[BINS];             // mass by bins, for top-p
    u64 chunk[1024];            // mass kept, by chunk of ids; without the cut's bin
    float lx[MANY];             // that bin's tokens
    int lid[MANY];
    u64 n_above;                // tokens kept, without the cut's bin
    u64 above, need;            // mass before that bin, mass that top-p asks for
    unsigned tops[MAX_PARTS];   // key of a slice's largest logit, ~0: a NaN or +inf
    unsigned n_list, first, done;   // first: the smallest id of the largest logit, where that one alone is kept
    Cut cut;
};

template <typename T>
struct Part {
    static constexpr int N = 16 / sizeof(T), CHUNK = 64 * N, AHEAD = 4;
    const T* x;
    int vocab, c0, c1;
    // f(chunk, id of the first, N logits) as Row's
    template <typename F>
    __device__ __forceinline__ void each_vec(F f) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        for (int c = c0 + wave; c < c1; c += PART_WAVES * AHEAD) {
            Some<T, N> s[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                s[j] = *reinterpret_cast<const Some<T, N>*>(x + min((c + j * PART_WAVES) * CHUNK + lane * N, vocab - N));
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int chunk = c + j * PART_WAVES;
                if (chunk >= c1) break;
                const int want = chunk * CHUNK + lane * N, i = min(want, vocab - N);
                float l[N];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    l[e] = q8_widen(s[j].v[e]);
                    l[e] = i + e >= want ? l[e] : -INFINITY;
                }
                f(chunk, i, l);
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ Part<T> part_of(const T* logits, int64_t ld, int vocab)
{
    const int n = (vocab + Part<T>::CHUNK - 1) / Part<T>::CHUNK, per = (n + gridDim.x - 1) / gridDim.x, c0 = blockIdx.x * per;
    return {logits + (size_t)blockIdx.y * ld, vocab, c0, min(c0 + per, n)};
}

// The row's masses; false: it has none
__device__ __forceinline__ bool masses_of(const Shared& g, int parts, float t0, Masses& m, unsigned& top)
{
    const int lane = threadIdx.x & 63;
    top = wave_max(lane < parts ? g.tops[lane] : 0u);
    m.top = logit_of(top);
    m.set(t0);
    return top != 0xffffffffu && m.top > -INFINITY;
}
__device__ __forceinline__ u64 least_mass(const float* min_p, int row)
{
    const float mp = min_p ? min_p[row] : 0.f;
    return mp > 0.f ? max((u64)ceil(fmin((double)mp, 1.0) * (double)MASS_ONE), (u64)1) : 1;
}

template <typename T>
__global__ void __launch_bounds__(PART_TPB) part_tops_kernel(const T* __restrict__ logits, int64_t ld, int vocab, Shared* __restrict__ shared)
{
    __shared__ unsigned tops[PART_WAVES];
    Shared& g = shared[blockIdx.y];
    unsigned top = 0;
    part_of(logits, ld, vocab).each_vec([&](int, int, const float* l) {
#pragma unroll
        for (int e = 0; e < Part<T>::N; ++e) top = max(top, l[e] < INFINITY ? key_of(l[e]) : 0xffffffffu);
    });
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    for (int i = blockIdx.x * PART_TPB + threadIdx.x; i < BINS; i += gridDim.x * PART_TPB) g.hist[i] = 0;
    __syncthreads();
    if (threadIdx.x) return;
    g.tops[blockIdx.x] = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    if (blockIdx.x == 0) {
        g.n_above = 0;
        g.n_list = 0;
        g.first = 0x7fffffffu;
    }
}

template <typename T>
__global__ void __launch_bounds__(PART_TPB) part_bins_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ temperature,
                                                             const float* __restrict__ top_p, Shared* __restrict__ shared)
{
    __shared__ u64 hist[BINS];
    Shared& g = shared[blockIdx.y];
    const float t0 = temperature ? temperature[blockIdx.y] : 1.f;
    Masses m;
    unsigned top;
    if (!masses_of(g, gridDim.x, t0, m, top) || !(t0 > 0.f) || !(top_p[blockIdx.y] < 1.f)) return;   // the workgroup as one
    for (int i = threadIdx.x; i < BINS; i += PART_TPB) hist[i] = 0;
    __syncthreads();
    part_of(logits, ld, vocab).each_vec([&](int, int, const float* l) {
#pragma unroll
        for (int e = 0; e < Part<T>::N; ++e) {
            const u64 w = m(l[e]);
            if (w) atomicAdd(&hist[m.bin(l[e])], w);
        }
    });
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += PART_TPB)
        if (hist[i]) atomicAdd(&g.hist[i], hist[i]);
}

// Mass kept, by chunk: of all bins before the one that top-p's cut falls into (without top-p of all), whose tokens are listed
template <typename T>
__global__ void __launch_bounds__(PART_TPB) part_masses_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ temperature,
                                                               const float* __restrict__ top_p, const float* __restrict__ min_p,
                                                               Shared* __restrict__ shared)
{
    __shared__ u64 waves[PART_WAVES];
    __shared__ int cut_bin;
    Shared& g = shared[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float t0 = temperature ? temperature[blockIdx.y] : 1.f, p = top_p ? top_p[blockIdx.y] : 1.f;
    const u64 least = least_mass(min_p, blockIdx.y);
    const Part<T> part = part_of(logits, ld, vocab);
    Masses m;
    unsigned top;
    if (!masses_of(g, gridDim.x, t0, m, top)) return;
    if (!(t0 > 0.f)) {   // the first token alone
        unsigned first = 0x7fffffffu;
        part.each_vec([&](int, int i0, const float* l) {
#pragma unroll
            for (int e = 0; e < Part<T>::N; ++e)
                if (l[e] == m.top) first = min(first, (unsigned)(i0 + e));
        });
        first = 0x7fffffffu - wave_max(0x7fffffffu - first);
        if (lane == 0 && first != 0x7fffffffu) atomicMin(&g.first, first);
        return;
    }
    int bin = BINS;
    if (p < 1.f) {
        constexpr int PER = BINS / PART_TPB;
        u64 h[PER], mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) mine += h[i] = g.hist[threadIdx.x * PER + i];
        const u64 upto = wave_scan(mine);
        if (lane == 63) waves[wave] = upto;
        if (threadIdx.x == 0) cut_bin = BINS;
        __syncthreads();
        u64 all = 0, before = upto - mine;
        for (int w = 0; w < PART_WAVES; ++w) {
            before += w < wave ? waves[w] : 0;
            all += waves[w];
        }
        const u64 need = share(p, all);
        if (before < need && before + mine >= need) {
            int i = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const bool on = i == k && before + h[k] < need;
                before += on ? h[k] : 0;
                i += on;
            }
            cut_bin = threadIdx.x * PER + i;
            if (blockIdx.x == 0) {
                g.above = before;
                g.need = need;
            }
        }
        __syncthreads();
        bin = cut_bin;
    }
    unsigned n = 0;
    part.each_vec([&](int chunk, int i0, const float* l) {
        unsigned hi = 0, lo = 0;   // of 512 masses at most: no carry out of either half
#pragma unroll
        for (int e = 0; e < Part<T>::N; ++e) {
            const u64 w = m(l[e]);
            const int b = bin < BINS ? w ? m.bin(l[e]) : BINS : 0;
            if (b == bin) {
                const unsigned at = atomicAdd(&g.n_list, 1u);
                if (at < MANY) {
                    g.lx[at] = l[e];
                    g.lid[at] = i0 + e;
                }
            }
            if (b >= bin || w < least) continue;
            ++n;
            hi += (unsigned)(w >> 22);
            lo += (unsigned)w & 0x3fffffu;
        }
        hi = wave_sum(hi);
        lo = wave_sum(lo);
        if (lane == 0) g.chunk[chunk] = ((u64)hi << 22) + lo;
    });
    n = wave_sum(n);
    if (lane == 0 && n) atomicAdd(&g.n_above, (u64)n);
}

// One workgroup a row: the cut within its bin, and the draw
template <typename T>
__global__ void __launch_bounds__(TPB) part_draw_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ uniforms,
                                                        const float* __restrict__ temperature, const float* __restrict__ top_p,
                                                        const float* __restrict__ min_p, int parts, int32_t* __restrict__ tokens,
                                                        float* __restrict__ logprob, int32_t* __restrict__ n_kept, float* __restrict__ out,
                                                        Shared* __restrict__ shared)
{
    constexpr int N = Part<T>::N, CHUNK = Part<T>::CHUNK;
    __shared__ Lds s;
    const int row = blockIdx.x, tid = threadIdx.x, n_chunks = (vocab + CHUNK - 1) / CHUNK;
    Shared& g = shared[row];
    // everything that the workspace has for this row, asked for at once: whether it is needed shows later
    const u64 chunk_mass = tid < n_chunks ? g.chunk[tid] : 0, n_above = g.n_above, above = g.above, need = g.need;
    const float t0 = temperature ? temperature[row] : 1.f, u = uniforms[row], first_l = g.lx[tid];
    const int n_list = (int)g.n_list, first_id = g.lid[tid];
    const Results o = {tokens + row, logprob ? logprob + row : nullptr, n_kept ? n_kept + row : nullptr, out ? out + (size_t)row * vocab : nullptr};
    const Params a = {0, top_p ? top_p[row] : 1.f, least_mass(min_p, row)};
    Masses m;
    unsigned top;
    const bool any = masses_of(g, parts, t0, m, top);
    if (!any || !(t0 > 0.f)) {
        if (tid == 0) {
            *o.token = any ? (int)g.first : -1;
            if (o.logprob) *o.logprob = any ? 0.f : __uint_as_float(0x7fc00000u);
            if (o.n_kept) *o.n_kept = any;
            g.cut = any ? Cut{top, (int)g.first} : Cut{0xffffffffu, -1};
            g.done = 0;
        }
        return;
    }
    Cut c = {0, vocab - 1};
    const int n = a.p < 1.f ? n_list : 0;
    if (n > MANY) {   // as many equal logits make
        slow_row<T, N>(logits + (size_t)row * ld, vocab, m, a, u, o, s);
        if (tid == 0) g.done = 1;
        return;
    }
    if (a.p < 1.f) {
        // each of the bin's tokens against each
        u64 *const order = s.hist, *const mass = s.hist + MANY;
        static_assert(2 * MANY <= BINS && MANY <= LIST, "the list's place");
        if (tid == 0) s.cut = c;
        const int n8 = (n + 7) & ~7;
        for (int i = tid; i < n8; i += TPB) {
            const float l = i >= n ? -INFINITY : i == tid ? first_l : g.lx[i];
            const int id = i >= n ? 0 : i == tid ? first_id : g.lid[i];
            s.lx[i] = l;
            s.lid[i] = id;
            order[i] = i < n ? order_of(l, id) : 0;
            mass[i] = m(l);
        }
        __syncthreads();
        for (int i = tid; i < n; i += TPB) {
            const u64 mine = order[i], upto = above + up_to(order, mass, n, mine);
            if (upto >= need && upto - mass[i] < need) s.cut = cut_at(mine);
        }
        __syncthreads();
        c = s.cut;
    }
    __syncthreads();
    s.hist[tid] = chunk_mass;
    static_assert(TPB == 1024, "a thread for each chunk");
    __syncthreads();
    u64 more = 0;
    for (int i = threadIdx.x; i < n; i += TPB) {
        const u64 w = m(s.lx[i]);
        if (w < a.least || !c.has(s.lx[i], s.lid[i])) continue;
        ++more;
        atomicAdd(&s.hist[s.lid[i] / CHUNK], w);
    }
    __syncthreads();
    Sums kept = block_sums(more, s.hist[tid], s);
    kept.n += n_above;
    draw_from_chunks<T, N>(logits + (size_t)row * ld, vocab, m, a, c, u, kept, o, s);
    if (threadIdx.x == 0) {
        g.cut = c;
        g.done = 0;
    }
}

template <typename T>
__global__ void __launch_bounds__(PART_TPB) part_write_kernel(const T* __restrict__ logits, int64_t ld, int vocab, const float* __restrict__ temperature,
                                                              const float* __restrict__ min_p, float* __restrict__ out,
                                                              const Shared* __restrict__ shared)
{
    constexpr int N = Part<T>::N;
    const Shared& g = shared[blockIdx.y];
    if (g.done) return;
    const float t0 = temperature ? temperature[blockIdx.y] : 1.f;
    const u64 least = t0 > 0.f ? least_mass(min_p, blockIdx.y) : 1;
    const Cut c = g.cut;
    Masses m;
    unsigned top;
    masses_of(g, gridDim.x, t0, m, top);
    float* const o = out + (size_t)blockIdx.y * vocab;
    part_of(logits, ld, vocab).each_vec([&](int chunk, int i0, const float* l) {
        const int want = (chunk * 64 + (int)(threadIdx.x & 63)) * N;
        Some<float, N> v;
#pragma unroll
        for (int e = 0; e < N; ++e) v.v[e] = l[e] > -INFINITY && c.has(l[e], i0 + e) && m(l[e]) >= least ? l[e] : -INFINITY;
        if (want + N <= vocab) *reinterpret_cast<Some<float, N>*>(o + i0) = v;
        else
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (i0 + e >= want && want < vocab) o[i0 + e] = v.v[e];
    });
}

// Workgroups a row; 1: the row is one workgroup's
int parts_of(int rows, int vocab, int dtype, bool top_p)
{
    // us, one workgroup a row and shared out, top-p 0.9: 1 row of 8192 29 and 22, of 32000 48 and 25, of 128256 160 and 27; 64 rows of 32000
    // 50 and 42, of 128256 168 and 70; 256 rows of 32000 58 and 71.  No filter: 1 row of 8192 14 and 15, of 32000 24 and 17, of
    // 128256 78 and 19; 64 rows of 128256 84 and 45, 256 rows 120 and 145.
    const int chunk = 64 * (dtype == SPEC_DTYPE_BF16 ? 8 : 4);
    if (vocab < (top_p ? 8192 : 16384) || rows > 128) return 1;
    return std::min(std::min(768 / rows, MAX_PARTS), vocab / (8 * chunk));
}

template <typename T>
void launch_parts(const spec_filter_args* a, const spec_filter_out* o, int parts, Shared* g, hipStream_t s)
{
    const T* x = (const T*)a->logits;
    const dim3 grid(parts, a->rows);
    hipLaunchKernelGGL((part_tops_kernel<T>), grid, dim3(PART_TPB), 0, s, x, a->ld, a->vocab, g);
    if (a->top_p) hipLaunchKernelGGL((part_bins_kernel<T>), grid, dim3(PART_TPB), 0, s, x, a->ld, a->vocab, a->temperature, a->top_p, g);
    hipLaunchKernelGGL((part_masses_kernel<T>), grid, dim3(PART_TPB), 0, s, x, a->ld, a->vocab, a->temperature, a->top_p, a->min_p, g);
    hipLaunchKernelGGL((part_draw_kernel<T>), dim3(a->rows), dim3(TPB), 0, s, x, a->ld, a->vocab, a->uniforms, a->temperature, a->top_p, a->min_p, parts,
                       o->tokens, o->logprob, o->n_kept, o->logits_out, g);
    if (o->logits_out) hipLaunchKernelGGL((part_write_kernel<T>), grid, dim3(PART_TPB), 0, s, x, a->ld, a->vocab, a->temperature, a->min_p, o->logits_out, g);
}

template <typename T, int NV, int N>
void launch_filter(const spec_filter_args* a, const spec_filter_out* o, hipStream_t s)
{
    hipLaunchKernelGGL((filter_kernel<T, NV, N>), dim3(a->rows), dim3(TPB), 0, s, (const T*)a->logits, a->ld, a->vocab, a->uniforms, a->temperature,
                       a->top_k, a->top_p, a->min_p, o->tokens, o->logprob, o->n_kept, o->logits_out);
}

template <typename T>
void launch_filter(const spec_filter_args* a, const spec_filter_out* o, hipStream_t s)
{
    constexpr int N = 16 / sizeof(T);
    // rows of up to 32768 logits stay in registers
    if (a->vocab < N) launch_filter<T, 1, 1>(a, o, s);
    else if (a->vocab <= 8192) launch_filter<T, 8192 / TPB / N, N>(a, o, s);
    else if (a->vocab <= 32768) launch_filter<T, 32768 / TPB / N, N>(a, o, s);
    else launch_filter<T, 0, N>(a, o, s);
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_filter_workspace_bytes(int32_t rows, int32_t vocab)
{
    // (of either type: fp32 rows are shared out among more workgroups)
    return rows > 0 && vocab > 0 && parts_of(rows, vocab, SPEC_DTYPE_FP32, true) > 1 ? (size_t)rows * sizeof(Shared) : 0;
}

extern "C" int spec_filter_sample(const spec_filter_args* a, const spec_filter_out* o, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || !o) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: null pointer");
    if (a->rows < 0 || a->vocab <= 0 || a->ld < a->vocab)
        return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: %d rows of %d logits, %lld elements apart", a->rows, a->vocab, (long long)a->ld);
    if (!q8_dtype(a->dtype)) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: unknown type %d", a->dtype);
    if (a->vocab > SPEC_FILTER_MAX_VOCAB) return fail(SPEC_ERR_SHAPE, "spec_filter_sample: vocabulary %d, at most %d", a->vocab, SPEC_FILTER_MAX_VOCAB);
    if (!a->rows) return SPEC_OK;
    if (!a->logits || !a->uniforms || !o->tokens) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: null pointer");
    if ((uintptr_t)workspace & 15) return fail(SPEC_ERR_INVALID_ARG, "spec_filter_sample: the workspace is not 16-byte aligned");
    const int parts = !a->top_k && workspace && workspace_bytes >= a->rows * sizeof(Shared) ? parts_of(a->rows, a->vocab, a->dtype, a->top_p != nullptr) : 1;
    const bool bf16 = a->dtype == SPEC_DTYPE_BF16;
    if (parts > 1 && bf16) launch_parts<uint16_t>(a, o, parts, (Shared*)workspace, (hipStream_t)stream);
    else if (parts > 1) launch_parts<float>(a, o, parts, (Shared*)workspace, (hipStream_t)stream);
    else if (bf16) launch_filter<uint16_t>(a, o, (hipStream_t)stream);
    else launch_filter<float>(a, o, (hipStream_t)stream);
    SPECV_LAUNCH_CHECK("filter_kernel");
    return SPEC_OK;
}
