// Causal attention over packed sequences.  The score product is S^T = K Q^T and the output O^T = V^T P^T, both by 32x32x16 matrix instructions: a
// lane then has one query row, whose maximum and sum it keeps in registers (the other half of the positions is lane ^ 32's), and the
// registers in which the score product leaves P^T are the ones that the second product takes it from, with the positions of 16 in the order
// 8 (e / 4) + 4 (lane / 32) + e % 4.  V^T comes out of LDS by transposing reads in the same order.
//
// A workgroup takes 32 WAVES query rows of one kv head, a row being one query head of one position: the query heads that share a kv head
// share its tile.  Keys and values pass through LDS in blocks of 64 positions, fetched one block ahead, once for all wavefronts.
//
// What bounds it: in long prompts the products, the exponentials beside them and the card's power -- 8192 positions of 32 heads of 128 517 to 530 us, 1.04 to
// 1.06 PFLOP/s, with zeros for operands 419; of 64, whose 32 exponentials stand beside half the products, 290 us, 0.95.  In short ones a tile's first fetch,
// its masked block and its end, some 11000 cycles beside 2000 a block: 16 prompts of 50 to 2100 of 32 heads of 64 146 us, 0.7 PFLOP/s, 160 in a loop of nothing
// else.  (Workgroups that stay for the next tile and look for it beside this one's first fetch: 171 where this took 154.)
#include "prompt.h"

#include <cfloat>

namespace specv {
namespace {

#define INLINE __attribute__((always_inline))   // (the kernel's lambdas: called, they would get scalars in vector registers)
constexpr int BLK = 64;   // positions of a block

struct Args {
    const uint16_t *q, *k, *v;
    uint16_t* out;
    int64_t ld_q, ld_k, ld_v, ld_out;
    const int32_t *q_row0, *k_row0;
    FastDiv heads, group;   // kv heads; query heads of one
    int batch, q_rows, k_rows;
    float factor;       // |scale| * log2(e), not zero: what is masked is -inf times it
    unsigned sign;      // 0x80008000 where the scale is negative: the queries are negated
    FastDiv parts;      // a tile's keys are shared out among at most so many workgroups,
    int chunk;          // each of which takes so many blocks (more where parts would not do); with more than one part, what they leave to the join:
    float *part_o, *part_ml;   // [unit][part][kv head][row of the tile][head_dim] sums of weighted values, [..][2] maximum and sum of weights
    bool by_place;      // the order of the tiles: by their place in their sequences, the last ones first; otherwise sequence by sequence
};

// The tile of a unit (its number and kv head): of one sequence, some rows.  Longer tiles come first, so that short ones fill what is left of the
// compute units' time: within a sequence, and with by_place over 64 sequences (8 x 1024 positions of 32 heads of 64: 57 -> 51 us; the search takes
// a microsecond more).
struct Tile {
    int seq, q_begin, n_q, k_begin, n_k, n_rows, row0;
};
template <int TILE>
__device__ __forceinline__ Tile find_tile(const Args& A, int number, bool by_place)
{
    const int group = A.group.d;
    PromptSpan q_span{0, 0}, k_span{0, 0};   // of the sequence that this lane looks at
    const PromptUnit unit = prompt_unit(number, A.batch, by_place, [&](int b) {
        q_span = k_span = prompt_span(A.q_row0, b, A.q_rows);
        if (A.k_row0) k_span = prompt_span(A.k_row0, b, A.k_rows);
        return ((q_span.end - q_span.begin) * group + TILE - 1) / TILE;
    });
    Tile t;
    t.seq = unit.seq;
    t.q_begin = __builtin_amdgcn_readlane(q_span.begin, unit.lane);
    t.n_q = __builtin_amdgcn_readlane(q_span.end, unit.lane) - t.q_begin;
    t.k_begin = __builtin_amdgcn_readlane(k_span.begin, unit.lane);
    t.n_k = __builtin_amdgcn_readlane(k_span.end, unit.lane) - t.k_begin;
    t.n_rows = t.n_q * group;
    t.row0 = unit.index * TILE;
    return t;
}

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
typedef __bf16 pr_bf16x2 __attribute__((ext_vector_type(2)));

// Blocks of a part, if the tile has that many in all
__device__ __forceinline__ int chunk_of(const Args& A, int all_blocks)
{
    return max(A.chunk, A.parts.div(all_blocks + (int)A.parts.d - 1));
}
// Blocks that some row of a tile sees
template <int TILE>
__device__ __forceinline__ int blocks_of(const Args& A, const Tile& T)
{
    const int last = T.n_k - T.n_q + A.group.div(min(T.row0 + TILE, T.n_rows) - 1);
    return last < 0 ? 0 : last / BLK + 1;
}

// A row of LDS holds the pieces (16 bytes) of a row of keys in the order piece ^ key_turn(row), of values piece ^ value_turn(row): the lanes that a
// read serves at once (sixteen of keys, 32 of values) then find different groups of banks
template <int HD>
__device__ __forceinline__ int key_turn(int r)
{
    return HD == 128 ? r & 15 : (r >> 1) & 7;
}
template <int HD>
__device__ __forceinline__ int value_turn(int r)
{
    return HD == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
}

// Position in the sequence and query head (of the kv head's) of a tile's row; rows beyond the last are the last again
__device__ __forceinline__ int2 place(const Args& A, const Tile& T, int row)
{
    row = min(T.row0 + row, T.n_rows - 1);
    const int at = A.group.div(row);
    return make_int2(at, row - at * (int)A.group.d);
}

// What a lane holds of the row `row` of its tile: to the output, or to the join
template <int HD, int TILE>
__device__ __forceinline__ void leave(const Args& A, const Tile& T, int head, int row, int half, const pr_floatx16 (&o)[HD / 32], float m, float sum, bool seen)
{
    if (T.row0 + row >= T.n_rows) return;
    if (A.parts.d > 1) {
        const size_t at = (size_t)blockIdx.x * TILE + row;      // (blockIdx.x counts kv heads, parts, units, in this order)
        float* po = A.part_o + at * HD + 4 * half;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<pr_floatx4*>(po + 32 * d + 2 * i) = (pr_floatx4){o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
        if (half == 0) *reinterpret_cast<float2*>(A.part_ml + 2 * at) = make_float2(m, sum);
        return;
    }
    const float inv = seen ? 1.f / sum : 0.f;
    const int2 to = place(A, T, row);
    // lane and lane ^ 32 exchange every other four dims: then each stores eight in a row
    uint16_t* dst = A.out + (size_t)(T.q_begin + to.x) * A.ld_out + (size_t)(head * (int)A.group.d + to.y) * HD + 8 * half;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            pr_uintx2 w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                w[j] = __builtin_amdgcn_permlane32_swap(pr_pack2(o[d][i + 2 * j] * inv, o[d][i + 2 * j + 1] * inv), pr_pack2(o[d][i + 4 + 2 * j] * inv, o[d][i + 5 + 2 * j] * inv),
                                                        false, false);
            *reinterpret_cast<pr_uintx4*>(dst + 32 * d + 2 * i) = (pr_uintx4){w[0][0], w[1][0], w[0][1], w[1][1]};
        }
}

// The lane's query row as operands of the score product
template <int HD>
__device__ __forceinline__ void load_query(const Args& A, const Tile& T, int head, int2 to, int half, pr_bf16x8 (&qf)[HD / 16])
{
    const uint16_t* src = A.q + (size_t)(T.q_begin + to.x) * A.ld_q + (size_t)(head * (int)A.group.d + to.y) * HD + 8 * half;
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) qf[c] = __builtin_bit_cast(pr_bf16x8, *reinterpret_cast<const pr_uintx4*>(src + 16 * c) ^ A.sign);
}

// Sixteen weights' worth of a lane: eight numbers exp2(s * factor - shift), rounded to bf16, and their sum (that of the rounded ones) added to l.  bf16
// because that is the values' type: with what the rounding leaves as a second operand the product with the values would be twice as long, half as much again of
// all products.  The result is 0.0020 of its size off (root mean square, 8192 positions), 0.0016 of it by its own rounding.
__device__ __forceinline__ pr_bf16x8 eight_weights(const pr_floatx16& s, int at, float factor, float shift, float& l)
{
    pr_uintx4 v;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[at + e], factor, -shift)), y = __builtin_amdgcn_exp2f(fmaf(s[at + e + 1], factor, -shift));
        unsigned both = pr_pack2(x, y);
        asm("" : "+v"(both));   // (a register of its own: as an element of v this compiler takes the first element's every time)
        l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pr_bf16x2, both), (pr_bf16x2){(__bf16)1.f, (__bf16)1.f}, l, false);
        v[e / 2] = both;
    }
    return __builtin_bit_cast(pr_bf16x8, v);
}

// Are there infinities or NaN among the KIB KiB of values at `part`?  (by one wavefront)
template <int KIB>
__device__ __forceinline__ bool has_odd(const char* part)
{
    unsigned any = 0;
#pragma unroll 2
    for (int i = 0; i < KIB; ++i) {
        const pr_uintx4 v = *reinterpret_cast<const pr_uintx4*>(part + (threadIdx.x & 63) * 16 + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7f807f80u) + 0x00800080u;
    }
    return __any((any & 0x80008000u) != 0);
}
// They leave the block's values (rows positions p0 ..); first: the positions of each column's first +infinity (NaN) and -infinity (NaN)
template <int HD, int ROWS>
__device__ __forceinline__ void clear_odd(char* part, int p0, int (*first)[HD], int tid, int threads)
{
#pragma unroll 1
    for (int d = tid; d < HD; d += threads) {
        int up = INT_MAX, down = INT_MAX;
#pragma unroll 1
        for (int r = ROWS - 1; r >= 0; --r) {
            uint16_t* const at = reinterpret_cast<uint16_t*>(part + r * (2 * HD) + ((d >> 3) ^ value_turn<HD>(r)) * 16) + (d & 7);
            const unsigned x = *at;
            if ((x & 0x7f80u) != 0x7f80u) continue;
            *at = 0;
            if ((x & 0x7fu) || !(x & 0x8000u)) up = p0 + r;
            if ((x & 0x7fu) || (x & 0x8000u)) down = p0 + r;
        }
        first[0][d] = up;
        first[1][d] = down;
    }
}
// Every row that sees the first one of a column has it in its sum
template <int HD>
__device__ __forceinline__ void add_odd(const int (*first)[HD], int half, int last, pr_floatx16 (&o)[HD / 32])
{
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int dim = 32 * d + 8 * (i / 4) + 4 * half + i % 4;
            o[d][i] += (first[0][dim] <= last ? INFINITY : 0.f) - (first[1][dim] <= last ? INFINITY : 0.f);
        }
}

template <int HD, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, HD == 64 && WAVES == 4 ? 3 : 2) attention_kernel(Args A)
{
    constexpr int ROW = 2 * HD, PART = BLK * ROW, KIB = PART / 1024;       // bytes of a row, of a block's keys; requests for them
    constexpr int PIECES = ROW / 16, ROWS = 1024 / ROW;                    // 16-byte pieces of a row, rows of a request
    constexpr int U = KIB / WAVES, TILE = 32 * WAVES;
    static_assert(KIB % WAVES == 0, "every wavefront has as many requests");
    __shared__ __attribute__((aligned(16))) char lds[4 * PART];            // keys, keys, values, values
    __shared__ int first[2][HD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r32 = lane & 31, half = lane >> 5;
    // Workgroups in a row take the kv heads: what they read lies together
    const int job = A.heads.div(blockIdx.x), head = (int)blockIdx.x - job * (int)A.heads.d, number = A.parts.div(job), part = job - number * (int)A.parts.d;
    const Tile T = find_tile<TILE>(A, number, A.by_place);
    if (T.seq < 0) return;
    const int last_first = T.n_k - T.n_q + A.group.div(T.row0), all_blocks = blocks_of<TILE>(A, T);
    // This part's blocks; all positions below are counted from their first one
    const int chunk = chunk_of(A, all_blocks), block0 = part * chunk, p_first = block0 * BLK;
    if (part && block0 >= all_blocks) return;
    const int n_blocks = min(all_blocks - block0, chunk);
    const int n_k = T.n_k - p_first, k_begin = T.k_begin + p_first;
    const int n_clear = last_first < p_first ? 0 : (last_first - p_first + 1) / BLK;       // blocks that all rows see whole

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const char* const kb = (const char*)(A.k + (size_t)k_begin * A.ld_k + (size_t)head * HD);
    const char* const vb = (const char*)(A.v + (size_t)k_begin * A.ld_v + (size_t)head * HD);
    uint32_t k_off[U], v_off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = (wave * U + u) * ROWS + lane / PIECES;
        k_off[u] = (uint32_t)r * (uint32_t)(2 * A.ld_k) + (lane % PIECES ^ key_turn<HD>(r)) * 16;
        v_off[u] = (uint32_t)r * (uint32_t)(2 * A.ld_v) + (lane % PIECES ^ value_turn<HD>(r)) * 16;
    }
    auto fetch_part = [&](const char* base, int64_t ld, const uint32_t (&off)[U], int block, uint32_t to, auto turn) INLINE {
        const int p0 = block * BLK;
        const char* from = base + (size_t)p0 * ld * 2;
        if (p0 + BLK <= n_k) {
#pragma unroll
            for (int u = 0; u < U; ++u) q8_fetch_lds(from, off[u], to + (wave * U + u) * 1024);
        } else {        // (beyond the end: the last row again)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = (wave * U + u) * ROWS + lane / PIECES;
                q8_fetch_lds(from, (uint32_t)min(r, n_k - 1 - p0) * (uint32_t)(2 * ld) + (lane % PIECES ^ turn(r)) * 16, to + (wave * U + u) * 1024);
            }
        }
    };
    auto fetch_keys = [&](int block) INLINE { fetch_part(kb, A.ld_k, k_off, block, lds0 + (block & 1) * PART, key_turn<HD>); };
    auto fetch_values = [&](int block) INLINE { fetch_part(vb, A.ld_v, v_off, block, lds0 + (2 + (block & 1)) * PART, value_turn<HD>); };

    if (n_blocks) {
        fetch_keys(0);
        fetch_values(0);
        if (n_blocks > 1) fetch_keys(1);
    }
    // (the fetches are under way) the lane's query row, and the last position that it sees
    const int2 to = place(A, T, wave * 32 + r32);
    const int last = n_k - T.n_q + to.x;
    pr_bf16x8 qf[HD / 16];
    load_query<HD>(A, T, head, to, half, qf);

    struct Scores {
        pr_floatx16 v[2];
    };
    pr_floatx16 o[HD / 32];
    Scores s0, s1;
    float m = -INFINITY, l[2] = {0.f, 0.f};   // (two sums, of even and of odd sixteens: one would be a chain of additions)
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

    // where this lane reads keys (rows r32, r32 + 32) and values (rows 4 half + (lane & 15) / 4 + 8 j)
    const int v_row = 4 * half + ((lane & 15) >> 2), v_turn = value_turn<HD>(v_row);
    auto key = [&](int par, int p, int c) INLINE {   // par: of the block's number, odd or even
        return *reinterpret_cast<const pr_bf16x8*>(lds + par * PART + (r32 + 32 * p) * ROW + ((2 * c + half) ^ key_turn<HD>(r32)) * 16);
    };
    auto value = [&](int par, int d, int k) INLINE {   // the operand of dims 32 d .. and positions 16 k ..
        const char* vl = lds + (2 + par) * PART + v_row * ROW + (lane & 1) * 8;
        const int piece = ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_turn) * 16;
        union {
            pr_shortx4 h[2];
            pr_bf16x8 f;
        } vf;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            vf.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pr_shortx4*)(vl + (16 * k + 8 * j) * ROW + piece));
        return vf.f;
    };
    auto scores = [&](Scores& t, int par, int p) INLINE {   // of positions 32 p .. 32 p + 31
#pragma unroll
        for (int i = 0; i < 16; ++i) t.v[p][i] = 0.f;
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) t.v[p] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key(par, p, c), qf[c], t.v[p], 0, 0, 0);
    };
    // The row's maximum over what it has seen, or an older one whose weights are larger by a factor of at most 2^8: the sums hold weights up to that as
    // well (rescaling at every new maximum: 8192 positions 533 us instead of 510)
    auto raise = [&](const Scores& s) INLINE {
        float top = fmaxf(s.v[0][0], s.v[0][1]);
#pragma unroll
        for (int i = 2; i < 32; i += 2) top = fmaxf(fmaxf(s.v[i / 16][i % 16], s.v[i / 16][i % 16 + 1]), top);
        top = both_max(top);
        const bool higher = (top - m) * A.factor > 8.f;
        if (__any(higher)) {
            const float up = higher ? top : m;      // (rows that need none keep theirs: their bits do not depend on the others' numbers)
            const float f = m == up ? 1.f : __builtin_amdgcn_exp2f((m - up) * A.factor);
            l[0] *= f;
            l[1] *= f;
#pragma unroll
            for (int d = 0; d < HD / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
            m = up;
        }
    };
    auto shift_of = [&]() { return m == -INFINITY ? 0.f : m * A.factor; };   // (a row that has seen nothing yet)
    auto weights = [&](const Scores& s, int k, float shift) INLINE { return eight_weights(s.v[k / 2], 8 * (k % 2), A.factor, shift, l[k & 1]); };   // of positions 16 k .. 16 k + 15
    auto sum_values = [&](int par, int k, pr_bf16x8 pf) INLINE {
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(par, d, k), pf, o[d], 0, 0, 0);
    };
    // Keys are fetched two blocks ahead and values one, in front of a block whose scores are there
    auto meet = [&](int block) INLINE {
        q8_wait_fetches<0>();
        q8_wait_lds();
        q8_barrier();
        if (block + 2 < n_blocks) fetch_keys(block + 2);
        if (block + 1 < n_blocks) fetch_values(block + 1);
    };
    // A block that all rows see whole, not the last one: the next block's scores, t, run beside this one's weights
    auto clear = [&](int block, auto par, const Scores& s, Scores& t) INLINE {
        constexpr int PAR = decltype(par)::value;
        meet(block);
        raise(s);
        const float shift = shift_of();
        const pr_bf16x8 p0 = weights(s, 0, shift);
        scores(t, 1 - PAR, 0);
        const pr_bf16x8 p1 = weights(s, 1, shift);
        scores(t, 1 - PAR, 1);
        const pr_bf16x8 p2 = weights(s, 2, shift);
        sum_values(PAR, 0, p0);
        const pr_bf16x8 p3 = weights(s, 3, shift);
        sum_values(PAR, 1, p1);
        sum_values(PAR, 2, p2);
        sum_values(PAR, 3, p3);
    };
    auto masked = [&](int block, Scores& s) INLINE {
        meet(block);
        const int seen = last - block * BLK - 4 * half;
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (8 * (i / 4) + i % 4 > seen) s.v[i / 16][i % 16] = -INFINITY;
        raise(s);
        // A weight of zero does not take an infinity or a NaN away
        char* const part = lds + (2 + (block & 1)) * PART;
        if (has_odd<KIB>(part)) {   // (every wavefront has looked at the same block, so all come here)
            q8_wait_lds();
            q8_barrier();
            clear_odd<HD, BLK>(part, block * BLK, first, threadIdx.x, 64 * WAVES);
            q8_wait_lds();
            q8_barrier();
            add_odd<HD>(first, half, last, o);
        }
        const float shift = shift_of();
#pragma unroll
        for (int k = 0; k < 4; ++k) sum_values(block & 1, k, weights(s, k, shift));
        if (block + 1 < n_blocks) {
            scores(s, 1 - (block & 1), 0);
            scores(s, 1 - (block & 1), 1);
        }
    };
    if (n_blocks) {
        q8_wait_fetches<0>();
        q8_barrier();
        scores(s0, 0, 0);
        scores(s0, 0, 1);
    }
    const int n_beside = min(n_clear, n_blocks - 1);
    int block = 0;
    for (; block + 1 < n_beside; block += 2) {
        clear(block, std::integral_constant<int, 0>(), s0, s1);
        clear(block + 1, std::integral_constant<int, 1>(), s1, s0);
    }
    if (block < n_beside) {
        clear(block++, std::integral_constant<int, 0>(), s0, s1);
        s0 = s1;
    }
    for (; block < n_blocks; ++block) masked(block, s0);
    const float sum = both_sum(l[0] + l[1]);
    int row = threadIdx.x;
    asm volatile("" : "+v"(row));   // (found anew: kept from above it would take registers all the way)
    const int own_half = (row >> 5) & 1;
    row = (row >> 6) * 32 + (row & 31);
    leave<HD, TILE>(A, T, head, row, own_half, o, m, sum, last >= 0);
}

// ---- few rows: the stream of keys and values -----------------------------------------------------------------------------
//
// One wavefront takes 32 query rows (those of a kv head's query heads at one position, say).  What bounds it is how much a compute unit has asked
// for at a time, so blocks are small, 32 positions, and go round in RING places of LDS of which all but one are under way.  More places leave room for
// fewer workgroups: 8 tokens behind 750 to 6000 positions, keys and values from memory, with the join 37, 35.6, 34.6, 35 us with 2, 3, 4, 5 places; from the card's
// last cache 24.2, 24.9, 25.8, 26.5; 64 behind 500 18.0, 16.4, 16.9, 17.4.
constexpr int FEW = 32, RING = 3;
template <int HD>
__global__ void __launch_bounds__(64, 1) few_kernel(Args A)
{
    constexpr int ROW = 2 * HD, PART = FEW * ROW, U = PART / 1024, PIECES = ROW / 16, ROWS = 1024 / ROW, TILE = 32;
    __shared__ __attribute__((aligned(16))) char lds[RING * 2 * PART];     // [place][keys, values]
    const int lane = threadIdx.x, r32 = lane & 31, half = lane >> 5;
    const int job = A.heads.div(blockIdx.x), head = (int)blockIdx.x - job * (int)A.heads.d, number = A.parts.div(job), part = job - number * (int)A.parts.d;
    const Tile T = find_tile<TILE>(A, number, false);
    if (T.seq < 0) return;
    const int all_blocks = blocks_of<TILE>(A, T), chunk = chunk_of(A, all_blocks), p_first = part * chunk * BLK;
    if (part && part * chunk >= all_blocks) return;
    // All positions are counted from the part's first one
    const int n_k = T.n_k - p_first, to_see = n_k - T.n_q;
    const int end = min(to_see + A.group.div(min(T.row0 + TILE, T.n_rows) - 1) + 1, min(all_blocks, chunk) * BLK);   // positions that some row sees
    const int n_blocks = end <= 0 ? 0 : (end + FEW - 1) / FEW, n_clear = to_see + A.group.div(T.row0) + 1;         // positions that all see

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const char* const kb = (const char*)(A.k + (size_t)(T.k_begin + p_first) * A.ld_k + (size_t)head * HD);
    const char* const vb = (const char*)(A.v + (size_t)(T.k_begin + p_first) * A.ld_v + (size_t)head * HD);
    auto fetch = [&](int block, int slot) INLINE {
        const int p0 = block * FEW;
        const char *kp = kb + (size_t)p0 * A.ld_k * 2, *vp = vb + (size_t)p0 * A.ld_v * 2;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = u * ROWS + lane / PIECES, from = min(r, n_k - 1 - p0);    // (beyond the end: the last row again)
            q8_fetch_lds(kp, (uint32_t)from * (uint32_t)(2 * A.ld_k) + (lane % PIECES ^ key_turn<HD>(r)) * 16, lds0 + slot * (2 * PART) + u * 1024);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = u * ROWS + lane / PIECES, from = min(r, n_k - 1 - p0);
            q8_fetch_lds(vp, (uint32_t)from * (uint32_t)(2 * A.ld_v) + (lane % PIECES ^ value_turn<HD>(r)) * 16, lds0 + slot * (2 * PART) + PART + u * 1024);
        }
    };
    for (int b = 0; b < min(n_blocks, RING - 1); ++b) fetch(b, b);
    const int2 to = place(A, T, r32);
    const int last = to_see + to.x;
    pr_bf16x8 qf[HD / 16];
    load_query<HD>(A, T, head, to, half, qf);

    pr_floatx16 o[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l[2] = {0.f, 0.f};
    const int v_row = 4 * half + ((lane & 15) >> 2), v_turn = value_turn<HD>(v_row);
    int slot = 0;
    for (int block = 0; block < n_blocks; ++block) {
        if (block + RING - 2 < n_blocks) q8_wait_fetches<(RING - 2) * 2 * U>();
        else q8_wait_fetches<0>();
        q8_wait_lds();
        if (block + RING - 1 < n_blocks) fetch(block + RING - 1, slot == 0 ? RING - 1 : slot - 1);
        char* const keys = lds + slot * (2 * PART);
        char* const values = keys + PART;
        pr_floatx16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) {
            const pr_bf16x8 kf = *reinterpret_cast<const pr_bf16x8*>(keys + r32 * ROW + ((2 * c + half) ^ key_turn<HD>(r32)) * 16);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[c], s, 0, 0, 0);
        }
        const bool masked = (block + 1) * FEW > n_clear;
        if (masked) {
            const int seen = last - block * FEW - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i / 4) + i % 4 > seen) s[i] = -INFINITY;
        }
        float top = fmaxf(s[0], s[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(s[i], s[i + 1]), top);
        top = fmaxf(both_max(top), m);
        if (__any(top > m)) {
            const float f = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * A.factor);
            l[0] *= f;
            l[1] *= f;
#pragma unroll
            for (int d = 0; d < HD / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
            m = top;
        }
        if (masked && has_odd<U>(values)) {
            int(*const first)[HD] = reinterpret_cast<int(*)[HD]>(keys);   // (the block's keys have been read)
            q8_wait_lds();
            clear_odd<HD, FEW>(values, block * FEW, first, lane, 64);
            q8_wait_lds();
            add_odd<HD>(first, half, last, o);
            q8_wait_lds();
        }
        const float shift = m == -INFINITY ? 0.f : m * A.factor;   // (a row that has seen nothing yet)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const pr_bf16x8 pf = eight_weights(s, 8 * k, A.factor, shift, l[k]);
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
                const int piece = ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_turn) * 16;
                union {
                    pr_shortx4 h[2];
                    pr_bf16x8 f;
                } vf;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    vf.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) pr_shortx4*)(values + (v_row + 16 * k + 8 * j) * ROW + (lane & 1) * 8 + piece));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.f, pf, o[d], 0, 0, 0);
            }
        }
        slot = slot == RING - 1 ? 0 : slot + 1;
    }
    leave<HD, TILE>(A, T, head, r32, half, o, m, both_sum(l[0] + l[1]), last >= 0);
}

// The parts of a tile's rows: eight dims of a row a thread, every fourth part a wavefront, whose sums meet in LDS (always in the same order).  Some 5 us, two
// round trips to memory among them.
template <int HD, int TILE>
__global__ void __launch_bounds__(256) join_kernel(Args A)
{
    constexpr int LANES = HD / 8, ROWS = 64 / LANES, GROUPS = TILE / ROWS;   // rows of a workgroup, workgroups of a tile
    const int job = blockIdx.x / GROUPS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = (blockIdx.x % GROUPS) * ROWS + lane / LANES, dim = lane % LANES * 8;
    const int number = A.heads.div(job), head = job - number * (int)A.heads.d, group = A.group.d;
    const Tile T = find_tile<TILE>(A, number, false);
    if (T.seq < 0 || T.row0 + (int)(blockIdx.x % GROUPS) * ROWS >= T.n_rows) return;
    const int blocks = blocks_of<TILE>(A, T), parts = max(1, (blocks + chunk_of(A, blocks) - 1) / chunk_of(A, blocks));
    const size_t step = (size_t)A.heads.d * TILE, first = ((size_t)number * A.parts.d * A.heads.d + head) * TILE + r;   // rows
    const float* ml = A.part_ml + first * 2;
    const float* po = A.part_o + first * HD + dim;
    float m = -INFINITY, l = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](float2 q, const pr_floatx4& a, const pr_floatx4& b) {
        const float top = fmaxf(m, q.x);
        const float old = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * A.factor), f = q.x == top ? 1.f : __builtin_amdgcn_exp2f((q.x - top) * A.factor);
        l = fmaf(q.y, f, l * old);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = fmaf(a[e], f, v[e] * old);
            v[4 + e] = fmaf(b[e], f, v[4 + e] * old);
        }
        m = top;
    };
    // eight parts at a time (beyond the last one: it again, not added): one by one each would wait for memory
    constexpr int N = 8;
    for (int p0 = wave; p0 < parts; p0 += 4 * N) {
        float2 q[N];
        pr_floatx4 a[N], b[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const size_t p = min(p0 + 4 * i, parts - 1);
            q[i] = *reinterpret_cast<const float2*>(ml + p * step * 2);
            a[i] = *reinterpret_cast<const pr_floatx4*>(po + p * step * HD);
            b[i] = *reinterpret_cast<const pr_floatx4*>(po + p * step * HD + 4);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (p0 + 4 * i < parts) add(q[i], a[i], b[i]);
    }
    __shared__ pr_floatx4 sums[4][2][64];
    __shared__ float2 tops[4][64];
    tops[wave][lane] = make_float2(m, l);
    sums[wave][0][lane] = (pr_floatx4){v[0], v[1], v[2], v[3]};
    sums[wave][1][lane] = (pr_floatx4){v[4], v[5], v[6], v[7]};
    __syncthreads();
    if (wave || T.row0 + r >= T.n_rows) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) add(tops[w][lane], sums[w][0][lane], sums[w][1][lane]);
    const int row = T.row0 + r, at = A.group.div(row), sub = row - at * group;
    const float inv = T.n_k - T.n_q + at < 0 ? 0.f : 1.f / l;
    pr_uintx4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pr_pack2(v[2 * i] * inv, v[2 * i + 1] * inv);
    *reinterpret_cast<pr_uintx4*>(A.out + (size_t)(T.q_begin + at) * A.ld_out + (size_t)(head * group + sub) * HD + dim) = w;
}

// How many wavefronts a workgroup has -- as many rows as the sequences have -- and how many blocks of keys: such that all of them together fill the
// places that the compute units have for workgroups at most once, and whatever of that takes least.  us: a block, with nothing to wait for but its
// predecessor (0.8 with heads of 64 and 1.35 of 128, a quarter more by one wavefront), the join's launch (5), the parts' way to memory and back.  Sequences
// differ in length: a tile may have several times as many parts as places allow on average.
constexpr int MOST_PARTS = 64;
struct Plan {
    int waves, parts, chunk;
    int64_t tiles;          // units of a launch, at most
    size_t part_bytes;      // of the workspace, for one part of every tile
    bool by_place;          // more workgroups than places
};
// (one wavefront: three workgroups of heads of 128 fit a compute unit, but places for four do better than for three or two -- 16 tokens behind up to 4000
// 45.7, 52, 46.5 us, 8 behind 6000 35.5, 35.4, 37.4 -- as shorter parts follow the ones that end first)
int64_t places_for(int waves, int head_dim) { return 256 * (waves == 1 ? 4 : head_dim == 128 ? 2 : waves == 4 ? 3 : 4); }
// of a tile, if one part of each of them makes wgs workgroups
int64_t most_parts(int waves, int head_dim, int64_t wgs) { return std::min((int64_t)MOST_PARTS, 4 / waves * places_for(waves, head_dim) / wgs); }
Plan plan(int q_rows, int k_rows, int batch, int n_kv_heads, int group, int head_dim, int64_t q_len, int64_t k_len, int waves = 0)
{
    Plan p;
    p.waves = waves ? waves : q_len * group <= 32 ? 1 : q_len * group <= 64 ? 2 : 4;
    const int rows = 32 * p.waves;
    p.tiles = (int64_t)q_rows * group / rows + batch;
    p.part_bytes = (size_t)p.tiles * n_kv_heads * rows * (head_dim + 2) * 4;
    const int64_t wgs = std::min(p.tiles, std::max((int64_t)batch, ((int64_t)q_rows * group + rows - 1) / rows)) * n_kv_heads;
    const int64_t places = places_for(p.waves, head_dim);
    const int64_t longest = (k_len + BLK - 1) / BLK, mean = std::min(longest, (int64_t)k_rows / batch / BLK + 1);
    const int64_t most = most_parts(p.waves, head_dim, wgs);
    // One sequence: as many parts of each tile as there are places.  Several, of different lengths: the last part of a tile is rarely a whole one, and
    // a few workgroups more than there are places take as long as twice as many.
    const int64_t each = std::max((int64_t)1, places / wgs), spare = std::max(places - wgs, places / 2);
    const int64_t least = std::max((int64_t)1, batch == 1 ? (longest + each - 1) / each : (wgs * mean + spare - 1) / spare);
    const float block = (p.waves == 1 ? 1.25f : 1.f) * (head_dim == 128 ? 1.35f : 0.8f), part = 2.f * (float)wgs * rows * (head_dim + 2) * 4 / 3.5e6f;
    int64_t chunk = longest;
    float us = block * (float)longest;
    for (int64_t n = 2; n <= most; n = n < most ? std::min(most, n + std::max((int64_t)1, n / 4)) : most + 1) {
        const int64_t c = std::max(least, (longest + n - 1) / n), parts = (longest + c - 1) / c;
        const float split = block * (float)c + 5.f + part * (float)parts;
        if (parts > 1 && split < us) us = split, chunk = c;
    }
    p.parts = (int)((longest + chunk - 1) / std::max((int64_t)1, chunk));
    if (p.parts < 1) p.parts = 1;
    p.chunk = (int)std::min(chunk, (int64_t)1 << 26);
    p.by_place = p.waves > 1 && batch > 1 && wgs > places;
    return p;
}

template <int HD, int WAVES>
void launch(const Args& a, const Plan& p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.tiles * a.heads.d * p.parts));
    if constexpr (WAVES == 1) hipLaunchKernelGGL((few_kernel<HD>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((attention_kernel<HD, WAVES>), grid, dim3(64 * WAVES), 0, s, a);
    if (p.parts > 1) {
        constexpr int GROUPS = 32 * WAVES * HD / 512;
        hipLaunchKernelGGL((join_kernel<HD, 32 * WAVES>), dim3((unsigned)(p.tiles * a.heads.d * GROUPS)), dim3(256), 0, s, a);
    }
}

}  // namespace
}  // namespace specv

using namespace specv;

extern "C" size_t spec_prompt_attention_workspace_bytes(int32_t q_rows, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (q_rows <= 0 || batch <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128)) return 0;
    size_t most = 0;
    for (int waves = 1; waves <= 4; waves *= 2) {
        const Plan p = plan(q_rows, INT_MAX, batch, n_kv_heads, n_q_heads / n_kv_heads, head_dim, 0, INT_MAX, waves);
        most = std::max(most, p.parts > 1 ? p.parts * p.part_bytes : 0);
    }
    return most;
}

extern "C" size_t spec_prompt_attention_workspace_bytes_up_to(int32_t q_rows, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (q_rows <= 0 || batch <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128)) return 0;
    size_t most = 0;
    for (int waves = 1; waves <= 4; waves *= 2) {
        // x: tiles that plan() counts on, the larger one of the sequences and of the tiles that the rows fill; a launch has those that the rows fill whole
        // and one for each sequence, x of both at most
        const int64_t rows = 32 * waves, whole = (int64_t)q_rows * (n_q_heads / n_kv_heads) / rows, all = std::max((int64_t)batch, whole + 1);
        for (int64_t x = 1; x <= all; ++x) {
            const int64_t parts = most_parts(waves, head_dim, x * n_kv_heads);
            if (parts < 2) break;
            most = std::max(most, (size_t)(parts * (std::min(x, whole) + std::min(x, (int64_t)batch)) * n_kv_heads * rows * (head_dim + 2) * 4));
        }
    }
    return most;
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
    const float factor = fabsf(a.scale) * 1.44269504088896341f;
    if (!(factor <= FLT_MAX)) return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: scale %g", (double)a.scale);
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
    if ((int64_t)a.q_rows * group > 0x3fffffff || ((int64_t)a.q_rows * group / 32 + a.batch) * a.n_kv_heads * 16 > 0x7fffffff)
        return fail(SPEC_ERR_SHAPE, "spec_prompt_attention: %d query rows are too many", a.q_rows);
    // (q_row0 is cut to the query rows, whatever it is read for)
    if (!a.k_row0 && a.k_rows != a.q_rows)
        return fail(SPEC_ERR_INVALID_ARG, "spec_prompt_attention: %d query rows, %d key rows and no k_row0", a.q_rows, a.k_rows);
    // lengths that are not known: all rows are of one sequence, or of as many as there are, whichever gives more workgroups
    const int64_t q_len = a.max_q_len ? a.max_q_len : a.q_rows, k_len = a.max_k_len ? a.max_k_len : a.k_rows;
    Plan p = plan(a.q_rows, a.k_rows, a.batch, a.n_kv_heads, group, a.head_dim, q_len, k_len);
    if (p.parts > 1) p.parts = workspace ? (int)std::min((size_t)p.parts, workspace_bytes / p.part_bytes) : 1;
    if (p.parts < 1) p.parts = 1;
    const int64_t units = p.tiles * a.n_kv_heads, threads = std::max(units * p.parts * 64 * p.waves, p.parts > 1 ? units * p.waves * a.head_dim * 16 : 0);
    if (threads > UINT32_MAX) return fail(SPEC_ERR_SHAPE, "spec_prompt_attention: %d query rows of %d sequences are too many for a launch", a.q_rows, a.batch);
    float* const ws = (float*)workspace;
    const size_t rows = p.part_bytes / (a.head_dim + 2) / 4 * p.parts;
    const Args g{(const uint16_t*)a.q, (const uint16_t*)a.k, (const uint16_t*)a.v, (uint16_t*)a.out, a.ld_q, a.ld_k, a.ld_v, a.ld_out, a.q_row0,
                 a.k_row0, FastDiv(a.n_kv_heads), FastDiv(group), a.batch, a.q_rows, a.k_rows, fmaxf(factor, 0x1p-149f),
                 a.scale < 0.f ? 0x80008000u : 0u, FastDiv(p.parts), p.parts > 1 ? p.chunk : 1 << 26, p.parts > 1 ? ws : nullptr, p.parts > 1 ? ws + rows * a.head_dim : nullptr, p.by_place && p.parts == 1};
    hipStream_t s = (hipStream_t)stream;
    if (a.head_dim == 128) {
        if (p.waves == 1) launch<128, 1>(g, p, s);
        else if (p.waves == 2) launch<128, 2>(g, p, s);
        else launch<128, 4>(g, p, s);
    } else {
        if (p.waves == 1) launch<64, 1>(g, p, s);
        else if (p.waves == 2) launch<64, 2>(g, p, s);
        else launch<64, 4>(g, p, s);
    }
    SPECV_LAUNCH_CHECK("attention_kernel");
    return SPEC_OK;
}
