// The rows of a prompt between two products: RMSNorm to bf16, rotary embedding with the cache's new entries.  Bound by memory.
#include "prompt.h"

#include "cache_layout.h"
#include "frag.h"
#include "handle.h"

namespace specv {
namespace {

constexpr int TPB = 256;

// Columns col .. col + 7 of a row (zero beyond cols)
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

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// W wavefronts take a row (W < 4: a workgroup takes 4 / W rows); a thread holds NV vectors of eight columns in registers between the sum of
// squares and the product with the gain, so the row is read once.  As many wavefronts as give a thread one vector, up to sixteen: all of a row is asked
// for at once.  4096 rows of 4096 fp32 16.5 us on buffers that the card's last cache holds in part, 19.7 on others, 5.1 TB/s (a copy's rate); one row of 2048
// 2.1 us on the GPU.
template <typename T, int W, int NV>
__global__ void __launch_bounds__(W < 4 ? 256 : 64 * W) rmsnorm_kernel(const T* __restrict__ x, const float* __restrict__ gain, uint16_t* __restrict__ y, int64_t ld, int rows,
                                                       int cols, float eps)
{
    constexpr int ROWS = W < 4 ? 4 / W : 1;
    __shared__ float part[W < 4 ? 4 : W];
    const int wave = threadIdx.x >> 6, sub = threadIdx.x % (64 * W);
    const int row = blockIdx.x * ROWS + wave / W;
    const bool live = row < rows;   // (all threads reach the barriers)
    const T* xr = x + (size_t)(live ? row : rows - 1) * ld;
    constexpr bool EARLY = NV <= 2;   // the gain is asked for with the row, while there are registers for both
    float h[NV][8], g[EARLY ? NV : 1][8], ss = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) load_cols(xr, (k * 64 * W + sub) * 8, cols, h[k]);
    if (EARLY) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_cols(gain, (k * 64 * W + sub) * 8, cols, g[EARLY ? k : 0]);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(h[k][i], h[k][i], ss);
    auto all = [&](float v, auto of_wave, auto join) {   // of the row, the same for all of its threads
        v = of_wave(v);
        if (W == 1) return v;
        if ((threadIdx.x & 63) == 0) part[wave] = v;
        __syncthreads();
        v = part[wave / W * W];
        for (int w = 1; w < W; ++w) v = join(v, part[wave / W * W + w]);
        return v;
    };
    auto add = [](float a, float b) { return a + b; };
    ss = all(ss, wave_sum, add);
    const float mean = ss / (float)cols + eps;
    float r = 1.f / sqrtf(mean);
    // Squares that leave fp32's range, and an eps beside which such squares count: the row over a power of two near its largest number, or eps's root if that is
    // larger, has others.  (Squares below 2^-126 lose bits; beside a sum of 2^-100 those do not count.  The barriers are the workgroup's: where some
    // row of it needs this, all do it, the others with the power 1.)
    const bool odd = !(ss <= 0x1.fffffep127f) || mean < 0x1p-100f;
    if (W == 1 ? (bool)__any(odd) : (bool)__syncthreads_or(odd)) {
        float top = sqrtf(eps);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(h[k][i]));
        if (W > 1) __syncthreads();
        top = all(top, wave_max, [](float a, float b) { return fmaxf(a, b); });
        const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252);   // (an infinity or a NaN leaves its mark in the sum below)
        const float down = odd ? __uint_as_float((unsigned)(254 - e) << 23) : 1.f;
        float s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[k][i] *= down;
                s2 = fmaf(h[k][i], h[k][i], s2);
            }
        if (W > 1) __syncthreads();
        s2 = all(s2, wave_sum, add);
        if (odd) r = 1.f / sqrtf(s2 / (float)cols + eps * down * down);
    }
    if (!live) return;
    uint16_t* yr = y + (size_t)row * cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * 64 * W + sub) * 8;
        if (col >= cols) continue;
        if (!EARLY) load_cols(gain, col, cols, g[0]);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = h[k][i] * r * g[EARLY ? k : 0][i];
        if (col + 8 <= cols) {
            pr_stream(yr + col, (pr_uintx4){pr_pack2(o[0], o[1]), pr_pack2(o[2], o[3]), pr_pack2(o[4], o[5]), pr_pack2(o[6], o[7])});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < cols) yr[col + i] = q8_round_bf16(o[i]);
        }
    }
}

template <typename T>
void launch_rmsnorm(const void* x, const float* gain, void* y, int64_t ld, int rows, int cols, float eps, hipStream_t s)
{
    auto go = [&](auto w, auto nv) {
        constexpr int W = decltype(w)::value, NV = decltype(nv)::value, ROWS = W < 4 ? 4 / W : 1;
        hipLaunchKernelGGL((rmsnorm_kernel<T, W, NV>), dim3((rows + ROWS - 1) / ROWS), dim3(W < 4 ? 256 : 64 * W), 0, s, (const T*)x, gain,
                           (uint16_t*)y, ld, rows, cols, eps);
    };
    auto n = [](auto v) { return v; };
#define N(V) n(std::integral_constant<int, V>())
    const int vecs = (cols + 7) / 8;
    if (vecs <= 64) go(N(1), N(1));
    else if (vecs <= 128) go(N(2), N(1));
    else if (vecs <= 256) go(N(4), N(1));
    else if (vecs <= 512) go(N(8), N(1));
    else if (vecs <= 1024) go(N(16), N(1));
    else if (vecs <= 2048) go(N(16), N(2));
    else if (vecs <= 4096) go(N(16), N(4));
    else go(N(16), N(8));
#undef N
}

// ---- rotary embedding, new keys and values ----------------------------------------------------------------------------

struct AppendArgs {
    CacheGeom g;
    const uint16_t* qkv;
    uint16_t *rotated, *cache;
    int64_t ld_qkv, ld_rot;
    const int32_t *row0, *seq_slot, *pos0;
    const float* cos_sin;
    int32_t* flag;
    int n_q_heads, layer, batch, rows, max_batch, max_kv_len, kv_blocks;
    FastDiv per_row, kv_heads;   // pairs of sixteen bytes of a row's queries; n_kv_heads
};

struct AppendSeq {
    int begin, len, slot, pos;
    bool ok;
};
__device__ __forceinline__ AppendSeq append_seq(const int32_t* row0, const int32_t* seq_slot, const int32_t* pos0, int b, int rows, int max_batch,
                                                int max_kv_len)
{
    const PromptSpan span = prompt_span(row0, b, rows);
    AppendSeq s{span.begin, span.end - span.begin, seq_slot[b], pos0 ? pos0[b] : 0, true};
    s.ok = s.slot >= 0 && s.slot < max_batch && s.pos >= 0 && s.pos <= max_kv_len - s.len;
    return s;
}

// Paged caches: pages up to the last new position of every slot.  The first sequence that names a slot covers for the others.  A thread walks a slot's pages
// one by one, in every layer's call: with this launch 37 rows of 32 heads of 128 take 10.8 us instead of 9.0, 1000 21.6 instead of 15.5, 8192 120 instead of 82.
__global__ void __launch_bounds__(64) append_cover_kernel(PagePool pool, const int32_t* __restrict__ row0, const int32_t* __restrict__ seq_slot, const int32_t* __restrict__ pos0, int batch,
                                    int rows, int max_batch, int max_kv_len, int32_t* flag)
{
    const int b = blockIdx.x * 64 + threadIdx.x;
    if (b >= batch) return;
    const AppendSeq s = append_seq(row0, seq_slot, pos0, b, rows, max_batch, max_kv_len);
    if (!s.ok || !s.len) return;
    int end = s.pos + s.len;
    for (int o = 0; o < batch; ++o) {
        if (o == b || seq_slot[o] != s.slot) continue;
        const AppendSeq t = append_seq(row0, seq_slot, pos0, o, rows, max_batch, max_kv_len);
        if (!t.ok || !t.len) continue;
        if (o < b) return;
        end = max(end, t.pos + t.len);
    }
    if (!pool_cover(pool, s.slot, 0, end)) atomicCAS(flag, 0, (int)SPEC_ERR_KV_OVERFLOW);
}

// Sixteen bytes of a row's head and the sixteen that they are paired with, rotated in fp32, rounded once
__device__ __forceinline__ void rotate8(pr_uintx4& a, pr_uintx4& b, const float* cs)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const pr_floatx4 c = *reinterpret_cast<const pr_floatx4*>(cs + 4 * i);   // cos, sin of two dims
        float lo[2], hi[2];
        rotate_pair(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), c[0], c[1], lo[0], hi[0]);
        rotate_pair(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), c[2], c[3], lo[1], hi[1]);
        a[i] = pr_pack2(lo[0], lo[1]);
        b[i] = pr_pack2(hi[0], hi[1]);
    }
}

// The first kv_blocks * n_kv_heads workgroups take one head of 32 positions of a sequence, as the cache has them in one block; the others 16
// rows' queries, 256 pairs of sixteen bytes at a time.  Memory bounds it: 6020 rows of 32 query and 32 kv heads of 128 80 to 82 us, 4.3 TB/s (a copy 5.1); four pairs
// of a thread asked for at once take 1 us off that, and a prompt of 37 rows then takes 6.3 us instead of 5.2.
template <int HD>
__global__ void __launch_bounds__(TPB) append_kernel(AppendArgs A)
{
    constexpr int PAIRS = HD / 16;      // of a row's head
    constexpr int LD = HD + 8;          // LDS row, 16-byte aligned
    const int n_kv = A.g.n_kv_heads;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < A.kv_blocks * n_kv) {
        __shared__ __align__(16) uint16_t values[32 * LD];
        const int block = A.kv_heads.div((int)blockIdx.x), head = (int)blockIdx.x - block * n_kv;
        const PromptUnit u = prompt_unit(block, A.batch, false, [&](int b) {
            const AppendSeq s = append_seq(A.row0, A.seq_slot, A.pos0, b, A.rows, A.max_batch, A.max_kv_len);
            if (!s.len) return 0;
            return s.ok ? ((s.pos + s.len - 1) >> 5) - (s.pos >> 5) + 1 : (s.len + 31) >> 5;
        });
        if (u.seq < 0) return;
        const AppendSeq s = append_seq(A.row0, A.seq_slot, A.pos0, u.seq, A.rows, A.max_batch, A.max_kv_len);
        const int base = s.ok ? ((s.pos >> 5) + u.index) << 5 : u.index << 5;       // position (row) of the unit's first place
        const int first = s.ok ? s.pos : 0;
        const int lo = max(first - base, 0), hi = min(first + s.len - base, 32);    // places of it that the sequence fills
        if (!s.ok && head == 0 && tid == 0 && u.index == 0)
            atomicCAS(A.flag, 0, s.slot < 0 || s.slot >= A.max_batch ? (int)SPEC_ERR_INVALID_ARG : (int)SPEC_ERR_KV_OVERFLOW);
        uint16_t* kc = nullptr;
        if (s.ok && !(A.g.table && A.g.table[(size_t)s.slot * A.g.blocks_per_slot + (base >> 5)] < 0))
            kc = A.cache + cache_block_base(A.g, A.layer, s.slot, head, base >> 5);
        // keys
        for (int i = tid; i < 32 * PAIRS; i += TPB) {
            const int t = i / PAIRS, p = i % PAIRS;
            if (t < lo || t >= hi) continue;
            const size_t row = (size_t)s.begin + (base + t - first);
            const uint16_t* src = A.qkv + row * A.ld_qkv + (size_t)(A.n_q_heads + head) * HD + 8 * p;
            pr_uintx4 a = *reinterpret_cast<const pr_uintx4*>(src), b = *reinterpret_cast<const pr_uintx4*>(src + HD / 2);
            if (s.ok) rotate8(a, b, A.cos_sin + (size_t)(base + t) * HD + 16 * p);
            else a = b = (pr_uintx4){0, 0, 0, 0};
            uint16_t* dst = A.rotated + row * A.ld_rot + (size_t)(A.n_q_heads + head) * HD + 8 * p;
            pr_stream(dst, a);
            pr_stream(dst + HD / 2, b);
            if (kc) {
                pr_stream(kc + tiled_k_within(HD, t, 8 * p), a);
                pr_stream(kc + tiled_k_within(HD, t, 8 * p + HD / 2), b);
            }
        }
        if (!kc) return;
        // values: a unit of the cache holds eight positions of one dim
        for (int i = tid; i < 32 * (HD / 8); i += TPB) {
            const int t = i / (HD / 8), c = i % (HD / 8) * 8;
            if (t < lo || t >= hi) continue;
            const size_t row = (size_t)s.begin + (base + t - first);
            *reinterpret_cast<pr_uintx4*>(values + t * LD + c) =
                *reinterpret_cast<const pr_uintx4*>(A.qkv + row * A.ld_qkv + (size_t)(A.n_q_heads + n_kv + head) * HD + c);
        }
        __syncthreads();
        for (int i = tid; i < 4 * HD; i += TPB) {
            const int lane = i & 63, dim = (i >> 6) * 16 + (lane & 15), g = lane >> 4;
            uint16_t e8[8];
            uint16_t* dst = kc + 32 * HD + (size_t)i * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) e8[e] = values[(e < 4 ? 4 * g + e : 12 + 4 * g + e) * LD + dim];
            if (lo == 0 && hi == 32) {
                pr_uintx4 v;
                __builtin_memcpy(&v, e8, 16);
                pr_stream(dst, v);
            } else {   // the block's other positions may hold entries: only these are written
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = e < 4 ? 4 * g + e : 12 + 4 * g + e;
                    if (t >= lo && t < hi) dst[e] = e8[e];
                }
            }
        }
        return;
    }
    // queries
    const int r0 = ((int)blockIdx.x - A.kv_blocks * n_kv) * 16;
    __shared__ int place[16];   // the row's position; -1: of a sequence that is skipped; -2: of none
    if (tid < 16) {
        int at = -2;
        const int row = r0 + tid;
        if (row < A.rows) {
            int lo = 0, hi = A.batch;   // the first sequence that ends behind the row
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (A.row0[mid + 1] <= row) lo = mid + 1;
                else hi = mid;
            }
            if (lo < A.batch) {
                const AppendSeq s = append_seq(A.row0, A.seq_slot, A.pos0, lo, A.rows, A.max_batch, A.max_kv_len);
                if (row >= s.begin) at = s.ok ? s.pos + (row - s.begin) : -1;
            }
        }
        place[tid] = at;
    }
    __syncthreads();
    const int per_row = A.per_row.d;
    for (int i = tid; i < 16 * per_row; i += TPB) {
        const int t = A.per_row.div(i), p = i - t * per_row, head = p / PAIRS, c = p % PAIRS * 8;
        const int at = place[t];
        if (at == -2) continue;
        const size_t row = (size_t)r0 + t;
        const uint16_t* src = A.qkv + row * A.ld_qkv + (size_t)head * HD + c;
        pr_uintx4 a = *reinterpret_cast<const pr_uintx4*>(src), b = *reinterpret_cast<const pr_uintx4*>(src + HD / 2);
        if (at >= 0) rotate8(a, b, A.cos_sin + (size_t)at * HD + 2 * c);
        else a = b = (pr_uintx4){0, 0, 0, 0};
        uint16_t* dst = A.rotated + row * A.ld_rot + (size_t)head * HD + c;
        pr_stream(dst, a);
        pr_stream(dst + HD / 2, b);
    }
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" int spec_prompt_rmsnorm(const void* x, int32_t x_dtype, int64_t ld, const float* gain, float eps, int32_t rows, int32_t cols, void* y,
                                   void* stream)
{
    if (rows < 0 || cols <= 0) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_rmsnorm: %d rows of %d columns", rows, cols);
    if (cols > SPEC_PROMPT_MAX_COLS) return fail(SPEC_ERR_SHAPE, "spec_prompt_rmsnorm: %d columns, at most %d", cols, SPEC_PROMPT_MAX_COLS);
    if (rows > SPEC_PROMPT_MAX_ROWS) return fail(SPEC_ERR_SHAPE, "spec_prompt_rmsnorm: %d rows, at most %d", rows, SPEC_PROMPT_MAX_ROWS);
    if (!q8_dtype(x_dtype)) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_rmsnorm: unknown type %d", x_dtype);
    if (ld < cols) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_rmsnorm: rows of %d columns are %lld elements apart", cols, (long long)ld);
    if (!(eps >= 0.f)) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_rmsnorm: eps %g", (double)eps);
    if (!rows) return SPEC_OK;
    if (!x || !gain || !y) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_rmsnorm: null pointer");
    if (x_dtype == SPEC_DTYPE_BF16) launch_rmsnorm<uint16_t>(x, gain, y, ld, rows, cols, eps, (hipStream_t)stream);
    else launch_rmsnorm<float>(x, gain, y, ld, rows, cols, eps, (hipStream_t)stream);
    SPECV_LAUNCH_CHECK("rmsnorm_kernel");
    return SPEC_OK;
}

extern "C" int spec_prompt_append(spec_handle* h, int32_t layer, const void* qkv, int64_t ld_qkv, void* rotated, int64_t ld_rotated,
                                  const int32_t* row0, const int32_t* seq_slot, const int32_t* pos0, int32_t batch, int32_t rows, void* stream)
{
    if (!h) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: NULL handle");
    if (!h->has_model) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: a sampler-only handle has no KV cache");
    const spec_model_cfg& c = h->cfg;
    if (c.dtype != SPEC_DTYPE_BF16) return fail(SPEC_ERR_SHAPE, "spec_prompt_append: bf16 models only");
    if (layer < 0 || layer >= c.n_layers) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: layer %d outside 0..%d", layer, c.n_layers - 1);
    if (batch < 0 || batch > c.max_batch || rows < 0)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: %d rows of %d sequences (at most %d)", rows, batch, c.max_batch);
    if (!batch || !rows) return SPEC_OK;
    if (!qkv || !rotated || !row0 || !seq_slot) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: null pointer");
    const int64_t cols = (int64_t)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, rot = (int64_t)(c.n_q_heads + c.n_kv_heads) * c.head_dim;
    if (ld_qkv < cols || ld_rotated < rot || ld_qkv % 8 || ld_rotated % 8 || ld_qkv > SPEC_PROMPT_MAX_LD || ld_rotated > SPEC_PROMPT_MAX_LD)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: rows %lld and %lld elements apart (at least %lld and %lld, multiples of 8, at most %d)",
                    (long long)ld_qkv, (long long)ld_rotated, (long long)cols, (long long)rot, SPEC_PROMPT_MAX_LD);
    if (((uintptr_t)qkv | (uintptr_t)rotated | (uintptr_t)h->kv_cache) & 15)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: qkv, rotated and the cache have to be 16-byte aligned");
    if (qkv == rotated && rows > 1 && ld_qkv != ld_rotated) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_append: in place with two different lds");
    const int64_t kv_blocks = std::min((int64_t)rows / 32 + 2 * (int64_t)batch, (int64_t)rows);   // a sequence of n rows reaches n / 32 + 2 blocks, and n at most
    const int64_t grid = kv_blocks * c.n_kv_heads + ((int64_t)rows + 15) / 16;
    if (grid * TPB > UINT32_MAX) return fail(SPEC_ERR_SHAPE, "spec_prompt_append: %d rows are too many", rows);
    hipStream_t s = (hipStream_t)stream;
    if (h->tables.pool.table) {
        hipLaunchKernelGGL(append_cover_kernel, dim3((batch + 63) / 64), dim3(64), 0, s, h->tables.pool, row0, seq_slot, pos0, batch, rows,
                           c.max_batch, c.max_kv_len, h->flag);
        SPECV_LAUNCH_CHECK("append_cover_kernel");
    }
    const AppendArgs a{h->geom, (const uint16_t*)qkv, (uint16_t*)rotated, (uint16_t*)h->kv_cache, ld_qkv, ld_rotated, row0, seq_slot, pos0,
                       h->cos_sin, h->flag, c.n_q_heads, layer, batch, rows, c.max_batch, c.max_kv_len, (int)kv_blocks,
                       FastDiv(c.n_q_heads * c.head_dim / 16), FastDiv(c.n_kv_heads)};
    if (c.head_dim == 128) hipLaunchKernelGGL((append_kernel<128>), dim3((unsigned)grid), dim3(TPB), 0, s, a);
    else hipLaunchKernelGGL((append_kernel<64>), dim3((unsigned)grid), dim3(TPB), 0, s, a);
    SPECV_LAUNCH_CHECK("append_kernel");
    return SPEC_OK;
}
