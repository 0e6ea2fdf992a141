// Device code of the 4-bit key / value cache (kg_op_kv4_*): append, read, attention over it, eviction.
//
// Format.  Per token, key / value head and group of 32 consecutive components: 16 levels,
//     m = fp16(min x),  s = fp16((max x - min x) / 15),  n = clamp(rint((x - m) / s), 0, 15),  value = s n + m,
// so 4 bits and a share of two halves: 5 bits a component, 3.2 times fewer bytes than fp16.  A group never spans tokens: a token is
// written, rolled back and moved (eviction) by itself, without touching its neighbours' numbers.
// Layout.  A physical page holds for each head one block of 5/4 T D bytes (T tokens, D components, G = D / 32 groups), laid out for the
// operands of v_mfma_f32_16x16x32_f16 (16 rows or columns x 32 products; lane = 16 q + row, 8 products per lane):
//     keys    [token][q of 4][g]          32-bit words, word (q, g) = components 32 g + 8 q + 0..7, lowest nibble first:
//                                         the 16 bytes of lane (token, q) are its products for all groups
//     values  [token / 4][r of 16][D / 64][token % 4]  16-bit words of nibbles i = components 16 (4 h + i) + r:
//                                         the 16 bytes of lane (r, q) hold four tokens, the products of probabilities and values
//     key scales [token / 4][g][token % 4], key minima [token][g], value scales, value minima [token / 4][g][token % 4], all fp16
#pragma once
#include "kernels.hip.h"

struct Kv4View {
    char *pool;
    size_t page_stride;
    const int *table, *len;
    int n_pages, logT, H, n_seqs, max_pages;
};

template <int D> struct Kv4 {
    static constexpr int G = D / 32, VH = D / 64;
    static __host__ __device__ constexpr int block(int T) { return T * D + T * D / 4; }
    // byte offsets in a head's block of a page of T tokens, token t of the page
    static __device__ __forceinline__ int k_word(int, int t, int q, int g) { return t * (D / 2) + (q * G + g) * 4; }
    static __device__ __forceinline__ int v_half(int T, int t, int r, int h) { return T * (D / 2) + ((((t >> 2) * 16 + r) * VH + h) * 4 + (t & 3)) * 2; }
    static __device__ __forceinline__ int quad(int t, int g) { return ((t >> 2) * G + g) * 8 + (t & 3) * 2; }
    static __device__ __forceinline__ int ks(int T, int t, int g) { return T * D + quad(t, g); }
    static __device__ __forceinline__ int km(int T, int t, int g) { return T * D + 2 * T * G + (t * G + g) * 2; }
    static __device__ __forceinline__ int vs(int T, int t, int g) { return T * D + 4 * T * G + quad(t, g); }
    static __device__ __forceinline__ int vm(int T, int t, int g) { return T * D + 6 * T * G + quad(t, g); }
};

// tokens of sequence s, as far as its page table reaches
__device__ __forceinline__ int kv4_len(const Kv4View &c, int s)
{
    const int n = c.len[s], cap = c.max_pages << c.logT;
    return n < 0 ? 0 : n > cap ? cap : n;
}
// the block of head h in the page of token t of sequence s; null where the table names no page of the pool
template <int D> __device__ __forceinline__ char *kv4_block(const Kv4View &c, int s, int h, int t)
{
    const int page = c.table[(size_t)s * c.max_pages + (t >> c.logT)];
    if (page < 0 || page >= c.n_pages) return nullptr;
    return c.pool + (size_t)page * c.page_stride + (size_t)h * Kv4<D>::block(1 << c.logT);
}

// The sequence of row r and the row's place in the cache (negative: rows of a sequence that is shorter than their number).
struct Kv4Row { int s, pos; };
__device__ __forceinline__ Kv4Row kv4_row(const Kv4View &c, const int *row_start, int r)
{
    int lo = 0, hi = c.n_seqs;                 // the last s with row_start[s] <= r
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row_start[mid] <= r) lo = mid; else hi = mid;
    }
    if (r < row_start[lo] || r >= row_start[lo + 1]) return {-1, 0};
    return {lo, kv4_len(c, lo) - row_start[lo + 1] + r};
}

// eight elements of a row
template <typename T> __device__ __forceinline__ void kv4_load8(const T *p, bool aligned, float (&x)[8])
{
    if (aligned) {
        typedef T vec_t __attribute__((ext_vector_type(8)));
        const vec_t v = *(const vec_t *)p;
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (float)p[e];
    }
}
template <typename T> __device__ __forceinline__ void kv4_store8(T *p, bool aligned, const float (&x)[8])
{
    if (aligned) {
        typedef T vec_t __attribute__((ext_vector_type(8)));
        vec_t v;
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (T)x[e];
        *(vec_t *)p = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) p[e] = (T)x[e];
    }
}
// are the rows' pieces of n elements all aligned for one access
template <typename T> __device__ __forceinline__ bool kv4_aligned(const void *p, long stride, int n)
{
    return (((uintptr_t)p | (uintptr_t)stride * sizeof(T)) & (n * sizeof(T) - 1)) == 0;
}

// The 16 levels of a group.  lo, hi: its least and largest component (clamped), bad: one of them is not finite.
struct Kv4Levels { float s, m, r; };            // r: 1 / s, 0 where every level is 0
__device__ __forceinline__ Kv4Levels kv4_levels(float lo, float hi, bool bad)
{
    Kv4Levels l;
    l.m = bad ? 0.f : (float)(_Float16)lo;
    l.s = bad ? __builtin_nanf("") : (float)(_Float16)__fdiv_rn(__fsub_rn(hi, lo), 15.f);
    l.r = l.s > 0.f ? __builtin_amdgcn_rcpf(l.s) : 0.f;
    return l;
}
// n = clamp(rint((x - m) / s), 0, 15) of the exact quotient.  (x - m) r in fp32 is within 4e-6 of it (three roundings of a number below 16,
// or beyond the last level), so only what comes as close as 1e-4 to a border is looked at again, in 64 bits, where x - m and n s are exact:
// one in 5000 (64 bits for all: 65 us instead of 39 for the append of 4096 rows of 32 heads).
__device__ __forceinline__ uint32_t kv4_level(float x, const Kv4Levels &l)
{
    const float t = fminf(fmaxf((x - l.m) * l.r, 0.f), 15.f);
    float n = rintf(t);
    if (fabsf(t - n) > 0.4999f) {
        const double s = l.s, rest = fma(-(double)n, s, (double)x - (double)l.m) * 2.0;
        const bool odd = (int)n & 1;
        if (rest > s || (rest == s && odd)) n += 1.f;
        else if (rest < -s || (rest == -s && odd)) n -= 1.f;
    }
    return (uint32_t)n;
}
__device__ __forceinline__ float kv4_clamp(float x) { return fminf(fmaxf(x, -65504.f), 65504.f); }
__device__ __forceinline__ bool kv4_bad(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// One row and head per D / 8 lanes, eight components each; a workgroup takes consecutive rows of one head, whose numbers lie together.
// Bound by the levels' arithmetic and the stores of two bytes, not by memory: 4096 bf16 rows of 32 heads (88 MB) 39 us, 2.3 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4View c, const T *k, long k_stride, const T *v, long v_stride, const int *row_start,
                                                         int n_rows)
{
    typedef Kv4<D> L;
    constexpr int LP = D / 8;
    const int li = threadIdx.x & (LP - 1), lane = threadIdx.x & 63, r = blockIdx.x * (256 / LP) + threadIdx.x / LP, h = blockIdx.y, P = 1 << c.logT;
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = y[e] = 0.f;
    // values: component 16 j + i, lane li has i = li (D = 128: j = 0..7) or i = li, li + 8 (D = 64: j = 0..3 each)
    if (r < n_rows) {
        kv4_load8(k + (size_t)r * k_stride + (size_t)h * D + 8 * li, kv4_aligned<T>(k, k_stride, 8), x);
        const T *row = v + (size_t)r * v_stride + (size_t)h * D + li;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = (float)row[D == 128 ? 16 * e : 16 * (e & 3) + 8 * (e >> 2)];
    }
    char *blk = nullptr;
    int t = 0;
    if (r < n_rows) {
        const Kv4Row row = kv4_row(c, row_start, r);
        if (row.s >= 0 && row.pos >= 0) {
            blk = kv4_block<D>(c, row.s, h, row.pos);
            t = row.pos & (P - 1);
        }
    }
    const bool live = blk != nullptr;
    {
        const int g = li >> 2, q = li & 3;
        float lo = INFINITY, hi = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            bad |= kv4_bad(x[e]);
            x[e] = kv4_clamp(x[e]);
            lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]);
        }
        lo = fminf(lo, quad_x1(lo)); hi = fmaxf(hi, quad_x1(hi));
        lo = fminf(lo, quad_x2(lo)); hi = fmaxf(hi, quad_x2(hi));
        const Kv4Levels l = kv4_levels(lo, hi, (__ballot(bad) >> (lane & ~3)) & 15);
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) w |= kv4_level(x[e], l) << (4 * e);
        if (live) {
            *(uint32_t *)(blk + L::k_word(P, t, q, g)) = w;
            if (q == 0) {
                *(_Float16 *)(blk + L::ks(P, t, g)) = (_Float16)l.s;
                *(_Float16 *)(blk + L::km(P, t, g)) = (_Float16)l.m;
            }
        }
    }
    bool bad[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        bad[e] = kv4_bad(y[e]);
        y[e] = kv4_clamp(y[e]);
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int g = 0; g < L::G; g++) {
        // the elements of group g: j = 2 g, 2 g + 1
        float lo = INFINITY, hi = -INFINITY;
        bool b = false;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if ((D == 128 ? e : e & 3) >> 1 != g) continue;
            lo = fminf(lo, y[e]); hi = fmaxf(hi, y[e]);
            b |= bad[e];
        }
        lo = fminf(lo, quad_x1(lo)); hi = fmaxf(hi, quad_x1(hi));
        lo = fminf(lo, quad_x2(lo)); hi = fmaxf(hi, quad_x2(hi));
        lo = fminf(lo, half_mirror(lo)); hi = fmaxf(hi, half_mirror(hi));
        if (LP == 16) { lo = fminf(lo, row_mirror(lo)); hi = fmaxf(hi, row_mirror(hi)); }
        const Kv4Levels l = kv4_levels(lo, hi, (__ballot(b) >> (lane & ~(LP - 1))) & ((1ull << LP) - 1));
#pragma unroll
        for (int e = 0; e < 8; e++) {
            if ((D == 128 ? e : e & 3) >> 1 != g) continue;
            w[e >> 2] |= kv4_level(y[e], l) << (4 * (e & 3));
        }
        if (live && li == g) {
            *(_Float16 *)(blk + L::vs(P, t, g)) = (_Float16)l.s;
            *(_Float16 *)(blk + L::vm(P, t, g)) = (_Float16)l.m;
        }
    }
    if (live) {
#pragma unroll
        for (int i = 0; i < 2; i++)
            *(uint16_t *)(blk + (D == 128 ? L::v_half(P, t, li, i) : L::v_half(P, t, li + 8 * i, 0))) = (uint16_t)w[i];
    }
}

// Keys and values of the rows, widened.  A token without a page reads as zeros.  Eight components of a row and head per lane.
// Bound by what it writes: 4096 rows of 32 heads to fp32 (155 MB) 30 us, 5.1 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4View c, T *k, long k_stride, T *v, long v_stride, const int *row_start, int n_rows)
{
    typedef Kv4<D> L;
    constexpr int LP = D / 8;
    const int li = threadIdx.x & (LP - 1), r = blockIdx.x * (256 / LP) + threadIdx.x / LP, h = blockIdx.y, P = 1 << c.logT;
    if (r >= n_rows) return;
    const Kv4Row row = kv4_row(c, row_start, r);
    if (row.s < 0 || row.pos < 0) return;
    const char *blk = kv4_block<D>(c, row.s, h, row.pos);
    const int t = row.pos & (P - 1), g = li >> 2, j = li >> 1;
    float kx[8] = {}, vx[8] = {};
    if (blk) {
        const uint32_t kw = *(const uint32_t *)(blk + L::k_word(P, t, li & 3, g));
        const float ks = (float)*(const _Float16 *)(blk + L::ks(P, t, g)), km = (float)*(const _Float16 *)(blk + L::km(P, t, g));
        const float vs = (float)*(const _Float16 *)(blk + L::vs(P, t, g)), vm = (float)*(const _Float16 *)(blk + L::vm(P, t, g));
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const uint32_t vw = *(const uint16_t *)(blk + L::v_half(P, t, 8 * (li & 1) + e, j >> 2));
            kx[e] = fmaf(ks, (float)(kw >> (4 * e) & 15), km);
            vx[e] = fmaf(vs, (float)(vw >> (4 * (j & 3)) & 15), vm);
        }
    }
    kv4_store8(k + (size_t)r * k_stride + (size_t)h * D + 8 * li, kv4_aligned<T>(k, k_stride, 8), kx);
    kv4_store8(v + (size_t)r * v_stride + (size_t)h * D + 8 * li, kv4_aligned<T>(v, v_stride, 8), vx);
}

// ---- attention ----------------------------------------------------------------------------------
//
// A column is one row and query head of a sequence and cache head.  A wave takes 4, 8 or 16 of them (few columns: decoding, verification) or 16 NC
// (many: prompts) over steps of 32 tokens (two tiles of 16).  What both kernels compute:
//   scores   z[t][c] = f_c (sum_g s_tg ((n_t - 8) . q_c)_g + (m_tg + 8 s_tg) (sum of q_c)_g): the levels are exact in fp16, so a group's 32 products are one
//            matrix instruction for each of two fp16 parts of the query (scaled by a power of two to below 2^10: the parts hold 24
//            bits), its scale a multiplication in fp32.  (Counted from the eighth, the sums that nearly cancel are half as large as from the first.)
//   softmax  over steps with a running reference M_c, the largest z_t + e_t seen, where the token's value scales are below 2^(e_t - 14):
//            2^(z - M + 28) s is then below 2^14 whatever the sizes of values and scales, and as two fp16 parts is held to 24 bits
//            and 2^-39 of the largest.
//   values   o[d][c] = sum_t (n_td - 8) (p_t s_tg)_c as matrix instructions, the levels again exact; sum_t p_t (m_tg + 8 s_tg) in fp32.
// With many columns the scores of a lane (column lane % 16, tokens 4 (lane / 16) + 0..3 of both tiles) are the products' side of the second
// matrix instruction, so probabilities never leave the lane, and the softmax and the values' operands are as said there.
struct Kv4Attn {
    Kv4View c;
    const void *q;
    void *out;
    long q_stride, out_stride;
    const int *row_start;
    int n_rows, heads, group, max_len;      // group: query heads of a cache head
    int chunk, n_chunks;                    // tokens of a workgroup; of the few-columns kernel a multiple of 128
    float scale, shift;                     // shift: the probabilities' factor 2^shift
    const float *w_in;
    float *w_out, *lse;                     // lse [row][head], base 2
    float *part;                            // [row][head][n_chunks][D]: a chunk's sums
    float2 *part_ml;                        // [row][head][n_chunks]: their reference, sum of the probabilities
};

constexpr float KV4_SHIFT = 28.f, KV4_MANY_SHIFT = 11.f;
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
union Kv4Op { uint32_t w[4]; f16x8_t v; };

// across the four lanes of a column
__device__ __forceinline__ float quads_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quads_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
// (w & mask) | bits in one instruction: the compiler makes two of it where both are constants
__device__ __forceinline__ f16x2_t and_or(uint32_t w, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(w), "s"(mask), "v"(bits));
    return __builtin_bit_cast(f16x2_t, r);
}
// levels i and i + 4 of a word as halves, less CENTRE, i = 0..3: 1024 + n, or 1024 + 16 n of the nibble above, less what is too much
template <int CENTRE = 0> __device__ __forceinline__ void kv4_widen(uint32_t w, uint32_t (&o)[4])
{
    const f16x2_t one = {(_Float16)(1024 + CENTRE), (_Float16)(1024 + CENTRE)}, sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const f16x2_t sixty_four = {(_Float16)(64 + CENTRE), (_Float16)(64 + CENTRE)};
    const uint32_t hi = w >> 8;
    o[0] = __builtin_bit_cast(uint32_t, and_or(w, 0x000f000fu, 0x64006400u) - one);
    o[1] = __builtin_bit_cast(uint32_t, and_or(w, 0x00f000f0u, 0x64006400u) * sixteenth - sixty_four);
    o[2] = __builtin_bit_cast(uint32_t, and_or(hi, 0x000f000fu, 0x64006400u) - one);
    o[3] = __builtin_bit_cast(uint32_t, and_or(hi, 0x00f000f0u, 0x64006400u) * sixteenth - sixty_four);
}
__device__ __forceinline__ float half_of(uint32_t w, int i) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(i ? w >> 16 : w)); }

// A pair of numbers as halves (one instruction), and in two parts, of which the second takes what the first leaves: 2^-24 of the number at
// most are lost.  (Parts rounded towards zero lose up to 2^-21, all to one side: outputs over 131001 tokens were off by 7.2e-6 instead of 2.1e-6, with levels counted from the first.)
__device__ __forceinline__ uint32_t kv4_halves(float x, float y) { return __builtin_bit_cast(uint32_t, f16x2_t{(_Float16)x, (_Float16)y}); }
__device__ __forceinline__ void kv4_split(float x, float y, uint32_t &hi, uint32_t &lo)
{
    float minus;                            // -1 in a register: x - (float)half as one mixed multiply-add, which the compiler would make a conversion and a difference
    asm("v_mov_b32 %0, -1.0" : "=v"(minus));
    asm("" : "+v"(x), "+v"(y));             // (numbers of fp32: a product that the compiler rounds to a half in one go would differ between instances)
    hi = kv4_halves(x, y);
    lo = kv4_halves(fmaf(half_of(hi, 0), minus, x), fmaf(half_of(hi, 1), minus, y));
}

// The columns of a block: sequence, first column, how many of the sequence's there are.
struct Kv4Cols { int s, c0, n, r0, end; };
template <int CB> __device__ __forceinline__ Kv4Cols kv4_columns(const Kv4Attn &a, int block)
{
    const int lane = threadIdx.x & 63;
    if (a.c.n_seqs == 1) {
        Kv4Cols k;
        const int first = a.row_start[0];
        k.s = 0; k.c0 = block * CB; k.end = a.row_start[1];
        k.r0 = min(max(first, 0), a.n_rows);
        k.n = (min(max(k.end, k.r0), a.n_rows) - k.r0) * a.group;
        if (k.c0 >= k.n) k.s = -1;
        return k;
    }
    int done = 0;
    for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) {
        const int s = s0 + lane;
        int r0 = 0, end = 0, rows = 0;
        if (s < a.c.n_seqs) {
            r0 = a.row_start[s]; end = a.row_start[s + 1];
            const int lo = min(max(r0, 0), a.n_rows);
            rows = min(max(end, lo), a.n_rows) - lo;
            r0 = lo;
        }
        const int nb = (rows * a.group + CB - 1) / CB;
        int sum = nb;
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(sum, o);
            if (lane >= o) sum += u;
        }
        const unsigned long long hit = __ballot(done + sum > block);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            Kv4Cols k;
            k.s = s0 + l;
            k.c0 = (block - done - __builtin_amdgcn_readlane(sum - nb, l)) * CB;
            k.n = __builtin_amdgcn_readlane(rows, l) * a.group;
            k.r0 = __builtin_amdgcn_readlane(r0, l);
            k.end = __builtin_amdgcn_readlane(end, l);
            return k;
        }
        done += __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0, 0, 0, 0};
}

// One column tile's queries: the products' side of the score instructions.  LO: the second part; 16-bit queries are exact without.
template <int D, bool LO> struct Kv4Query {
    Kv4Op hi[D / 32], lo[LO ? D / 32 : 1], sum;      // slot 2 i, 2 i + 1 of lane group q: components 8 q + i, 8 q + i + 4 of the group
    float total[4];                         // the groups' sums of the queries, scaled as the parts
    float f;                                // what a sum of products is worth as a base-2 exponent: not negative, the scale's sign is in the parts

    // CENTRE: the first parts of the sums in lane group 1 too, against the second parts of m + 8 s (Kv4Ops)
    template <bool CENTRE = false, typename T> __device__ __forceinline__ void load(const T *row, bool live, bool aligned, float scale, int q)
    {
        constexpr int G = D / 32;
        float x[G][8], mx = 0.f;
#pragma unroll
        for (int g = 0; g < G; g++) {
#pragma unroll
            for (int e = 0; e < 8; e++) x[g][e] = 0.f;
            if (live) kv4_load8(row + 32 * g + 8 * q, aligned, x[g]);
#pragma unroll
            for (int e = 0; e < 8; e++) mx = fmaxf(mx, fabsf(x[g][e]));
        }
        mx = quads_max(mx);
        const int ex = mx > 0.f && mx <= 3.402823466e38f ? __builtin_amdgcn_frexp_expf(mx) : 10;
        f = fmaxf(__builtin_amdgcn_ldexpf(fabsf(scale) * 1.44269504088896341f, ex - 10), 1.17549435e-38f);     // (above 0: a masked score stays -inf)
        const float sign = scale < 0.f ? -1.f : 1.f;
        uint32_t sh[2] = {0, 0}, sl[2] = {0, 0};
        total[0] = total[1] = total[2] = total[3] = 0.f;
#pragma unroll
        for (int g = 0; g < G; g++) {
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) { x[g][e] = __builtin_amdgcn_ldexpf(x[g][e] * sign, 10 - ex); t += x[g][e]; }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (LO) kv4_split(x[g][i], x[g][i + 4], hi[g].w[i], lo[LO ? g : 0].w[i]);
                else hi[g].w[i] = kv4_halves(x[g][i], x[g][i + 4]);
            }
            total[g] = quads_sum(t);
        }
        kv4_split(total[0], total[1], sh[0], sl[0]);
        kv4_split(total[2], total[3], sh[1], sl[1]);
        sum.w[0] = q <= (CENTRE ? 1 : 0) ? sh[0] : 0; sum.w[1] = q <= (CENTRE ? 1 : 0) ? sh[1] : 0;       // groups 0..3 against the minima's slots 0..3 and 4..7
        sum.w[2] = q == 0 ? sl[0] : 0; sum.w[3] = q == 0 ? sl[1] : 0;
    }
};

// A step's numbers in LDS, brought there without passing registers (lds_load16: 16 bytes a lane, lane after lane, from any addresses):
// keys of both tiles as their readers want them, values likewise, then for each tile its parts of the four tables.
template <int D> struct Kv4Stage {
    static constexpr int G = D / 32, LOADS = D == 128 ? 5 : 3, BYTES = LOADS * 1024;
    static __device__ __forceinline__ int k_read(int i, int lane)
    {
        return D == 128 ? i * 1024 + lane * 16 : i * 512 + ((lane & 15) + (lane >> 5) * 16) * 16 + (lane >> 4 & 1) * 8;
    }
    static __device__ __forceinline__ int v_read(int i, int lane) { return D == 128 ? 2048 + i * 1024 + lane * 16 : 1024 + i * 512 + lane * 8; }
    static __device__ __forceinline__ int table(int i, int n) { return D == 128 ? 4096 + i * 512 + n * 128 : 2048 + i * 256 + n * 64; }
    // load n of the LOADS of a step: blocks b0, b1 of the tiles and their first tokens t0, t1 in the page
    static __device__ __forceinline__ void load(int n, const char *b0, int t0, const char *b1, int t1, int P, uint32_t lds, int lane)
    {
        if (D == 128) {
            const char *b = n & 1 ? b1 : b0;
            const int t = n & 1 ? t1 : t0;
            if (n < 2) lds_load16(b + t * 64, (lane & 15) * 64 + (lane >> 4) * 16, lds + n * 1024);
            else if (n < 4) lds_load16(b + P * 64 + t * 64, lane * 16, lds + n * 1024);
            else {
                const char *x = lane < 32 ? b0 + t0 * 8 : b1 + t1 * 8;
                lds_load16(x + P * D + (lane >> 3 & 3) * 8 * P + (lane & 7) * 16, lds + 4096);
            }
        } else {
            const int l = lane & 31;
            if (n == 0) lds_load16((lane < 32 ? b0 + t0 * 32 : b1 + t1 * 32) + (l & 15) * 32 + (l >> 4) * 16, lds);
            else if (n == 1) lds_load16((lane < 32 ? b0 + t0 * 32 : b1 + t1 * 32) + P * 32 + l * 16, lds + 1024);
            else {              // 32 lanes' worth; the others repeat them behind
                const char *x = (l < 16 ? b0 + t0 * 4 : b1 + t1 * 4);
                lds_load16(x + P * D + (l >> 2 & 3) * 4 * P + (l & 3) * 16, lds + 2048);
            }
        }
    }
};
// until at most n loads are under way
template <int N> __device__ __forceinline__ void loads_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// what was read from LDS has arrived: the place may be written again
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The numbers of one tile of 16 tokens as they lie in the page.
template <int D> struct Kv4Keys {
    static constexpr int G = D / 32;
    uint32_t w[G], s[2 * G], m[G / 2];      // lane's token: words; tokens 4 q + 0..3: scales; lane's token: minima

    // tile of tokens t.. of a page
    __device__ __forceinline__ void load_page(const char *blk, int P, int t, int lane)
    {
        const uint32_t q = lane >> 4, tok = lane & 15;
        __builtin_memcpy(w, __builtin_assume_aligned(blk + Kv4<D>::k_word(P, t, 0, 0) + (tok * (D / 2) + q * 4 * G), 4 * G), 4 * G);
        __builtin_memcpy(s, __builtin_assume_aligned(blk + Kv4<D>::ks(P, t, 0) + q * 8 * G, 16), 8 * G);
        __builtin_memcpy(m, __builtin_assume_aligned(blk + Kv4<D>::km(P, t, 0) + tok * 2 * G, 2 * G), 2 * G);
    }
    // tile i of a step in LDS (Kv4Stage)
    __device__ __forceinline__ void load(const char *stage, int i, int lane)
    {
        const int q = lane >> 4, tok = lane & 15;
        __builtin_memcpy(w, __builtin_assume_aligned(stage + Kv4Stage<D>::k_read(i, lane), 4 * G), 4 * G);
        __builtin_memcpy(s, __builtin_assume_aligned(stage + Kv4Stage<D>::table(i, 0) + q * 8 * G, 16), 8 * G);
        __builtin_memcpy(m, __builtin_assume_aligned(stage + Kv4Stage<D>::table(i, 1) + tok * 2 * G, 2 * G), 2 * G);
    }
    // the levels as the other side of the score instructions
    template <int CENTRE = 0> __device__ __forceinline__ void widen(f16x8_t (&k)[G]) const
    {
#pragma unroll
        for (int g = 0; g < G; g++) {
            Kv4Op o;
            kv4_widen<CENTRE>(w[g], o.w);
            k[g] = o.v;
        }
    }
    // scores of tokens 4 q + 0..3 in the units of Kv4Query::f
    template <bool LO> __device__ __forceinline__ f32x4_t scores(const f16x8_t (&k)[G], const Kv4Query<D, LO> &x) const
    {
        Kv4Op mm;
        mm.w[0] = mm.w[2] = m[0];
        mm.w[1] = mm.w[3] = G == 4 ? m[G / 2 - 1] : 0;
        const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
        f32x4_t z = __builtin_amdgcn_mfma_f32_16x16x32_f16(mm.v, x.sum.v, zero, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < G; g++) {
            f32x4_t d = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[g], x.hi[g].v, zero, 0, 0, 0);
            if (LO) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[g], x.lo[LO ? g : 0].v, d, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; i++) z[i] = fmaf(half_of(s[2 * g + (i >> 1)], i & 1), d[i], z[i]);
        }
        return z;
    }
};
template <int N> __device__ __forceinline__ void lds_read(uint32_t (&x)[N], const char *p)
{
    __builtin_memcpy(x, __builtin_assume_aligned(p, N >= 4 ? 16 : 4 * N), 4 * N);
}
// what comes behind is not begun before what stands in front: keeps the numbers of a later part of a step out of the registers
#define KV4_PART __builtin_amdgcn_sched_barrier(0)

// The step's two tiles: where they lie (null: no page, none of its tokens is seen).
struct Kv4Step { const char *blk[2]; int t[2]; bool here[2]; };
template <int D> __device__ __forceinline__ Kv4Step kv4_step(const Kv4View &c, int s, int h, int t0, int limit)
{
    Kv4Step st;
    const int P = 1 << c.logT;
    // (constant memory while the kernel runs: scalar loads, which do not queue behind the loads that fill the LDS)
    const __attribute__((address_space(4))) int *table = (const __attribute__((address_space(4))) int *)(c.table + (size_t)s * c.max_pages);
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int t = t0 + 16 * i;
        int page = -1;
        if (t < limit) page = table[t >> c.logT];
        st.here[i] = page >= 0 && page < c.n_pages;
        st.t[i] = st.here[i] ? t & (P - 1) : 0;                 // (a tile that is not there is read as page 0 and masked)
        st.blk[i] = c.pool + (size_t)(st.here[i] ? page : 0) * c.page_stride + (size_t)h * Kv4<D>::block(P);
    }
    return st;
}

// Keeps all four registers of a matrix instruction's result until y, which was computed from it, is there.  The compiler gives the registers of
// numbers that nobody reads to other values at once, with too short a distance: the instruction's late write then destroyed these (scores of
// all groups from the third on were wrong).
__device__ __forceinline__ void whole_until(float &y, const f32x4_t &d) { asm("" : "+v"(y) : "v"(d)); }

// Few columns: a wave's state for 4 NV of them.  The scores' matrix has the columns (queries) as rows and the tokens as columns: column
// c is row 4 (c % 4) + c / 4, so that lane (q, token) holds the scores of columns q, q + 4, .. (NV of them) with its own token of each tile:
// with one or four columns no lane computes an exponential or splits a product for a column that is not there.  The probabilities
// times the values' scales go through LDS (xchg) to the lanes that multiply them: products 2 j, 2 j + 1 of lane group q are tokens 4 q + j of
// both tiles.
//   Bound by memory where the cache is long: one row of 32 heads over 131001 tokens (671 MB) 130 to 146 us by the card, 5.2 to 4.6 TB/s (a plain read
//   of memory: 6.5); 158 us against the 130 where every lane held 16 columns.  Levels counted from the eighth cost 2 % of that and leave
//   8.8e-7 of error for 2.1e-6.  Short caches are a chain of latencies: 500 tokens 6.2 us of which 0.5 is memory.
template <int D, int NV> struct Kv4Few {
    static constexpr int G = D / 32, DT = D / 16, VH = D / 64, C = 4 * NV;
    static constexpr int XCHG = G * 2 * C * 64;         // bytes: [group][part][column][16 tokens] pairs of halves
    f32x4_t o[DT];                              // column lane % 16 (modulo C), d = 16 j + 4 q + 0..3
    float om[NV][G], m[NV], l[NV];              // columns q + 4 i; om and l: the lane's tokens' part

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int j = 0; j < DT; j++) o[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
#pragma unroll
            for (int g = 0; g < G; g++) om[i][g] = 0.f;
            m[i] = -INFINITY; l[i] = 0.f;
        }
    }
    // One step of 32 tokens from t0 on, its numbers in LDS.  MASK: lim[i] is the number of tokens that the lane's columns see, here: the tiles that
    // have a page.  Written so that few of the step's numbers are in registers at a time.
    template <bool MASK, bool LO>
    __device__ __forceinline__ void step(const Kv4Query<D, LO> &x, const float (&qs)[NV][G], const float (&f)[NV], const char *stage, char *xchg,
                                         const int (&lim)[NV], int here, int t0, int lane)
    {
#pragma clang fp contract(off)                      // (all instances round alike: a row's bits do not depend on which one it went through)
        typedef Kv4Stage<D> S;
        const int q = lane >> 4, tok = lane & 15;
        const auto number = [&](int i, int table, int g) {      // of the lane's token in tile i
            return (float)*(const _Float16 *)(stage + S::table(i, table) + ((tok >> 2) * G + g) * 8 + (tok & 3) * 2);
        };
        float z[2][NV];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            Kv4Keys<D> k;
            k.load(stage, i, lane);
            f16x8_t kk[G];
            k.template widen<8>(kk);
            const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
            float y[NV];
#pragma unroll
            for (int g = 0; g < G; g++) {
                f32x4_t d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.hi[g].v, kk[g], zero, 0, 0, 0);
                if (LO) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.lo[LO ? g : 0].v, kk[g], d, 0, 0, 0);
                const float s = number(i, 0, g), mid = fmaf(s, 8.f, half_of(k.m[g >> 1], g & 1));
#pragma unroll
                for (int n = 0; n < NV; n++) y[n] = fmaf(s, d[n], g == 0 ? mid * qs[n][0] : fmaf(mid, qs[n][g], y[n]));
                whole_until(y[NV - 1], d);
            }
#pragma unroll
            for (int n = 0; n < NV; n++) z[i][n] = y[n] * f[n];
        }
        KV4_PART;
        float vs[2][G], e[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            // s < 2^(e - 14) for all groups of the token (of garbage: e is some number).  Scales are not negative: halves compare as whole numbers
            uint32_t mx = 0;
#pragma unroll
            for (int g = 0; g < G; g++) {
                const _Float16 v = *(const _Float16 *)(stage + S::table(i, 2) + ((tok >> 2) * G + g) * 8 + (tok & 3) * 2);
                vs[i][g] = (float)v;
                mx = max(mx, (uint32_t)__builtin_bit_cast(uint16_t, v));
            }
            e[i] = (float)(mx >> 10 & 31);
        }
        bool see[2][NV];
        float p[2][NV], mx[NV];
        bool grows = false;
#pragma unroll
        for (int n = 0; n < NV; n++) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                see[i][n] = !MASK || ((here >> i & 1) && t0 + 16 * i + tok < lim[n]);
                if (!see[i][n]) z[i][n] = -INFINITY;
            }
            mx[n] = row_max(fmaxf(z[0][n] + e[0], z[1][n] + e[1]));
            grows |= mx[n] > m[n];
        }
        if (__any(grows)) {                         // (where a column's stays its factor is 1)
            float alpha[NV], to = 0.f;
#pragma unroll
            for (int n = 0; n < NV; n++) {
                const float m_new = fmaxf(m[n], mx[n]);
                alpha[n] = __builtin_amdgcn_exp2f(m[n] - (m_new == -INFINITY ? 0.f : m_new));
                l[n] *= alpha[n];
                m[n] = m_new;
#pragma unroll
                for (int g = 0; g < G; g++) om[n][g] *= alpha[n];
                const float v = __shfl(alpha[n], 16 * (tok & 3));       // of column tok, if that is one of these four
                to = ((tok & (C - 1)) >> 2) == n ? v : to;
            }
#pragma unroll
            for (int j = 0; j < DT; j++) o[j] *= to;
        }
#pragma unroll
        for (int n = 0; n < NV; n++) {
            const float ref = (m[n] == -INFINITY ? 0.f : m[n]) - KV4_SHIFT;
#pragma unroll
            for (int i = 0; i < 2; i++) p[i][n] = __builtin_amdgcn_exp2f(z[i][n] - ref);
            l[n] += p[0][n] + p[1][n];
#pragma unroll
            for (int g = 0; g < G; g++) {
                const float x0 = see[0][n] ? p[0][n] * vs[0][g] : 0.f, x1 = see[1][n] ? p[1][n] * vs[1][g] : 0.f;
                uint32_t hi, lo;
                kv4_split(x0, x1, hi, lo);
                char *at = xchg + ((g * 2) * C + q + 4 * n) * 64 + tok * 4;
                __builtin_memcpy(__builtin_assume_aligned(at, 4), &hi, 4);         // (not as words: what reads them reads halves, and has to come behind)
                __builtin_memcpy(__builtin_assume_aligned(at + C * 64, 4), &lo, 4);
            }
        }
#pragma unroll
        for (int g = 0; g < G; g++) {
            const float m0 = fmaf(vs[0][g], 8.f, number(0, 3, g)), m1 = fmaf(vs[1][g], 8.f, number(1, 3, g));
#pragma unroll
            for (int n = 0; n < NV; n++) {
                const float y0 = fmaf(p[0][n], m0, om[n][g]);
                om[n][g] = see[0][n] ? y0 : om[n][g];
                const float y1 = fmaf(p[1][n], m1, om[n][g]);
                om[n][g] = see[1][n] ? y1 : om[n][g];
            }
        }
        KV4_PART;
        uint32_t vw[2][2 * VH];
#pragma unroll
        for (int i = 0; i < 2; i++) lds_read(vw[i], stage + S::v_read(i, lane));
#pragma unroll
        for (int h = 0; h < VH; h++) {
            uint32_t u[4][4];                       // token 4 q + j of both tiles: nibbles i
#pragma unroll
            for (int a = 0; a < 2; a++) {
                const uint32_t w0 = vw[0][2 * h + a], w1 = vw[1][2 * h + a];
                kv4_widen<8>((w0 & 0xffff) | w1 << 16, u[2 * a]);
                kv4_widen<8>(w0 >> 16 | (w1 & 0xffff0000u), u[2 * a + 1]);
            }
#pragma unroll
            for (int g = 2 * h; g < 2 * h + 2; g++) {
                Kv4Op hi, lo;
                const char *at = xchg + ((g * 2) * C + (tok & (C - 1))) * 64 + q * 16;
                lds_read(hi.w, at);
                lds_read(lo.w, at + C * 64);
#pragma unroll
                for (int j = 2 * g; j < 2 * g + 2; j++) {
                    Kv4Op a;
#pragma unroll
                    for (int w = 0; w < 4; w++) a.w[w] = u[w][j & 3];
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, hi.v, o[j], 0, 0, 0);
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, lo.v, o[j], 0, 0, 0);
                }
            }
        }
    }
};

// Steps t0, t0 + stride, .. below t1, by one wave with a ring of NS steps in LDS of its own: NS - 1 are under way while one is
// worked on.  start() before the queries are loaded.
template <int D, int NS> struct Kv4Ring {
    static constexpr int S = Kv4Stage<D>::LOADS, B = Kv4Stage<D>::BYTES;
    const Kv4View &c;
    const char *lds;
    int s, h, t1, stride, lane;
    int here;                                   // two bits per step of the ring, the next step's lowest: its tiles that have a page
    __device__ __forceinline__ void fetch(int slot, int ahead, int t)
    {
        const Kv4Step st = kv4_step<D>(c, s, h, t, t1);
        here |= (st.here[0] | st.here[1] << 1) << (2 * ahead);
        const uint32_t at = lds_address(lds) + slot * B;
#pragma unroll
        for (int n = 0; n < S; n++) Kv4Stage<D>::load(n, st.blk[0], st.t[0], st.blk[1], st.t[1], 1 << c.logT, at, lane);
    }
    __device__ __forceinline__ void start(int t0)
    {
        here = 0;
#pragma unroll
        for (int i = 0; i < NS - 1; i++)
            if (t0 + i * stride < t1) fetch(i, i, t0 + i * stride);
    }
    template <int NV, bool LO>
    __device__ __forceinline__ void run(Kv4Few<D, NV> &state, const Kv4Query<D, LO> &x, const float (&qs)[NV][D / 32], const float (&f)[NV], char *xchg,
                                        const int (&lim)[NV], int least, int t0)
    {
        int slot = 0;
        for (int t = t0; t < t1; t += stride) {
            lds_reads_done();
            if (t + (NS - 1) * stride < t1) {
                fetch(slot == 0 ? NS - 1 : slot - 1, NS - 1, t + (NS - 1) * stride);
                loads_left<(NS - 1) * S>();
            } else if (NS > 2 && t + (NS - 2) * stride < t1) loads_left<(NS - 2) * S>();
            else loads_left<0>();
            const char *stage = lds + slot * B;
            if (t + 32 <= least && (here & 3) == 3) state.template step<false, LO>(x, qs, f, stage, xchg, lim, here, t, lane);
            else state.template step<true, LO>(x, qs, f, stage, xchg, lim, here, t, lane);
            here >>= 2;
            slot = slot == NS - 1 ? 0 : slot + 1;
        }
    }
};

// what a lane's column is: row and head, tokens it sees (0: a column behind the sequence's last)
struct Kv4Column { int row, head, lim; };
__device__ __forceinline__ Kv4Column kv4_column(const Kv4Attn &a, const Kv4Cols &k, int h, int col, int len)
{
    Kv4Column c;
    const bool live = col < k.n;
    const int i = live ? col : 0;
    c.row = k.r0 + i / a.group;
    c.head = h * a.group + i % a.group;
    c.lim = live ? max(0, min(len - k.end + c.row + 1, a.max_len)) : 0;
    return c;
}
// the same for a column that is the wave's
__device__ __forceinline__ int kv4_row_lim(const Kv4Attn &a, const Kv4Cols &k, int col, int len)
{
    return max(0, min(len - k.end + k.r0 + col / a.group + 1, a.max_len));
}
// outputs d = 16 j + 4 q + 0..3 of a row, from sums over l
template <typename T> __device__ __forceinline__ void kv4_store4(T *p, bool aligned, f32x4_t v)
{
    if (aligned) {
        typedef T vec_t __attribute__((ext_vector_type(4)));
        *(vec_t *)p = vec_t{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = (T)v[i];
    }
}

// Few columns: a workgroup takes a chunk of the tokens for one cache head and up to 4 NV columns, its four waves every fourth step.  (Rings of three
// steps, two for 16 columns: two workgroups a compute unit.)
template <typename T, int D, int NV>
__global__ __launch_bounds__(256, 2) void kv4_attend_few_kernel(const Kv4Attn a)
{
    constexpr int G = D / 32, DT = D / 16, C = 4 * NV, NS = NV == 4 ? 2 : 3, RING = NS * Kv4Stage<D>::BYTES, XCHG = Kv4Few<D, NV>::XCHG;
    constexpr bool LO = sizeof(T) == 4;
    __shared__ __align__(16) char ring[4 * RING], xchg[4 * XCHG];
    __shared__ float ms[4][C], ls[4][C], oms[4][C][G];
    float (*os)[C][D + 4] = (float (*)[C][D + 4])ring;      // after the steps: the waves' sums
    static_assert(sizeof(float[4][C][D + 4]) <= 4 * RING, "the waves' sums fit the rings");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, h = blockIdx.y, chunk = blockIdx.z;
    const Kv4Cols k = kv4_columns<C>(a, blockIdx.x);
    if (k.s < 0) return;
    const int len = kv4_len(a.c, k.s);
    const int most = kv4_row_lim(a, k, min(k.c0 + C, k.n) - 1, len), least = kv4_row_lim(a, k, k.c0, len);     // (later columns see no less)
    const int t0 = chunk * a.chunk, t1 = min(most, t0 + a.chunk);
    if (t0 >= t1 && chunk > 0) return;                    // the merge knows from the rows' places
    Kv4Ring<D, NS> steps = {a.c, ring + wave * RING, k.s, h, t1, 128, lane, 0};
    steps.start(t0 + 32 * wave);
    // row lane % 16 of the scores' matrix is column (lane % 16) / 4 + 4 (lane % 4)
    const int c = (lane >> 2 & 3) + 4 * (lane & 3);
    const bool live = c < C && k.c0 + c < k.n;
    const Kv4Column col = kv4_column(a, k, h, k.c0 + c, live ? len : 0);
    Kv4Query<D, LO> x;
    x.load((const T *)a.q + (size_t)col.row * a.q_stride + (size_t)col.head * D, live, kv4_aligned<T>(a.q, a.q_stride, 8), a.scale, q);
    // a lane's scores are of columns q, q + 4, ..: rows 4 q, 4 q + 1, ..
    float f[NV], qs[NV][G];
    int lim[NV];
#pragma unroll
    for (int n = 0; n < NV; n++) {
#pragma unroll
        for (int g = 0; g < G; g++) qs[n][g] = __shfl(x.total[g], 4 * q + n);
        f[n] = __shfl(x.f, 4 * q + n);
        lim[n] = __shfl(live ? col.lim : 0, 4 * q + n);
    }
    Kv4Few<D, NV> state;
    state.clear();
    steps.run(state, x, qs, f, xchg + wave * XCHG, lim, least, t0 + 32 * wave);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NV; n++) {
        const float l = row_sum(state.l[n]);
        if ((lane & 15) == 0) { ms[wave][q + 4 * n] = state.m[n]; ls[wave][q + 4 * n] = l; }
#pragma unroll
        for (int g = 0; g < G; g++) {
            const float v = row_sum(state.om[n][g]);
            if ((lane & 15) == 0) oms[wave][q + 4 * n][g] = v;
        }
    }
    if ((lane & 15) < C)
#pragma unroll
        for (int j = 0; j < DT; j++) *(f32x4_t *)&os[wave][lane & 15][16 * j + 4 * q] = state.o[j];
    __syncthreads();
    // a thread takes four outputs of a column
    for (int i = threadIdx.x; i < C * (D / 4); i += 256) {
        const int cc = i / (D / 4), d = i % (D / 4) * 4;
        if (k.c0 + cc >= k.n) continue;
        const Kv4Column kc = kv4_column(a, k, h, k.c0 + cc, len);
        float m = ms[0][cc];
        for (int w = 1; w < 4; w++) m = fmaxf(m, ms[w][cc]);
        const float ref = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < 4; w++) {
            const float fw = __builtin_amdgcn_exp2f(ms[w][cc] - ref), om = oms[w][cc][d >> 5];
            l = fmaf(fw, ls[w][cc], l);
            const f32x4_t ow = *(const f32x4_t *)&os[w][cc][d];
            for (int e = 0; e < 4; e++) o[e] = fmaf(fw, ow[e] + om, o[e]);
        }
        if (a.n_chunks > 1) {
            const size_t at = ((size_t)kc.row * a.heads + kc.head) * a.n_chunks + chunk;
            *(f32x4_t *)(a.part + at * D + d) = o;
            if (d == 0) a.part_ml[at] = float2{m, l};
        } else {
            for (int e = 0; e < 4; e++) o[e] = l == 0.f ? 0.f : o[e] / l;
            kv4_store4((T *)a.out + (size_t)kc.row * a.out_stride + (size_t)kc.head * D + d, kv4_aligned<T>(a.out, a.out_stride, 4), o);
            if (d == 0) a.lse[(size_t)kc.row * a.heads + kc.head] = l == 0.f ? -INFINITY : m - a.shift + __builtin_amdgcn_logf(l);
        }
    }
}

// Many columns (prompt rows): a workgroup takes 64 NC columns of a cache head over the tokens of a chunk, a wave 16 NC of them.  What a step of
// 32 tokens is multiplied with is made once per workgroup, by all four waves, in LDS: the keys' levels (the scores' scales stay a
// multiplication in fp32), and the values so that the probabilities need no group's scale: 8 of them per step and lane, not 8 G.
//   fp32 and fp16 rows: the values as two exact fp16 parts, n s = n (s's upper 7 bits) + n (its lower 4 bits), the minima as one more
//     instruction over the probabilities, these in two parts.  Of the four products fp16 rows leave out that of both second parts (2^-18).
//     Levels are counted from the eighth, minima from there too (m + 8 s, in two parts): the sums that nearly cancel are half as large, and so is
//     the error (scores off by 4.7e-6 instead of 9.6e-6, 30 their size; 6.1e-6 where keys are widened first and then multiplied in fp32).
//   bf16 rows: values s n + m and probabilities rounded to fp16, 2^-11 each of what they are, an eighth of the 2^-8 that the output is rounded by:
//     half of the matrix instructions and of what is read from LDS.
// Steps with a scale of 2048 or a minimum of 16384 or more take a sixteenth of the values (they might not fit a half) and 16 p.
// A value scale that is not a number counts as 0 here and makes the outputs of the columns that see it NaN (nan).
//   2048 bf16 rows of 32 heads behind 4096 tokens (172 GFLOP): 461 us, 373 TFLOP/s, a third of a large library product.  A step's matrix
//   instructions (154 us in all) and vector instructions (218 us) follow one another at two waves a SIMD; tiles of 16 or 64 columns a wave,
//   rings of two or four steps and three waves a SIMD (which spill) were no faster.
template <int D> struct Kv4Ops {                // byte offsets of a step's operands, 16 bytes a lane each
    static constexpr int G = D / 32, DT = D / 16, K = 0, VHI = 2 * G * 1024, VLO = VHI + DT * 1024, VM = VLO + DT * 1024, KM = VM + 1024;
    static constexpr int bytes(bool parts) { return parts ? KM + 2 * 1024 : VLO; }
};
struct Kv4Scales { bool big, nan; };            // of a step's value scales: big as above, one that is not a number

// Which of a step's tokens count: `left` from its first on, and of those the ones in tiles that have a page (bits of `there`).
struct Kv4Part {
    int left, there;
    __device__ __forceinline__ bool all() const { return left >= 32 && there == 3; }
    __device__ __forceinline__ int end(int i) const { return there >> i & 1 ? left - 16 * i : 0; }      // of tile i
};
// tokens of a pair t, t + 1 that count, as a mask of halves
__device__ __forceinline__ uint32_t kv4_pair_mask(int t, int end) { return (t < end ? 0xffffu : 0u) | (t + 1 < end ? 0xffff0000u : 0u); }
template <int D> __device__ __forceinline__ Kv4Scales kv4_scales(const char *stage, const Kv4Part &part, int lane)
{
    constexpr int G = D / 32, WORDS = 8 * G;    // of a tile
    const int l = lane & (2 * WORDS - 1), i = l / WORDS, n = l % WORDS;
    uint32_t w = *(const uint32_t *)(stage + Kv4Stage<D>::table(i, 2) + 4 * n), m = *(const uint32_t *)(stage + Kv4Stage<D>::table(i, 3) + 4 * n);
    if (!part.all()) {
        const uint32_t mask = kv4_pair_mask(n / (2 * G) * 4 + (n & 1) * 2, i ? part.end(1) : part.end(0));
        w &= mask; m &= mask;
    }
    // halves as whole numbers: 2048 is 0x6800, 16384 0x7400, infinity 0x7c00 and what is not a number beyond
    const uint32_t lo = w & 0x7fff, hi = w >> 16 & 0x7fff, ml = m & 0x7fff, mh = m >> 16 & 0x7fff;
    Kv4Scales r = {false, false};
    if (__any(max(lo, hi) >= 0x6800 || max(ml, mh) >= 0x7400)) {
        r.nan = __any(lo > 0x7c00 || hi > 0x7c00);
        r.big = __any((lo >= 0x6800 && lo <= 0x7c00) || (hi >= 0x6800 && hi <= 0x7c00) || max(ml, mh) >= 0x7400);
    }
    return r;
}
__device__ __forceinline__ uint32_t kv4_nan_to_zero(uint32_t w)
{
    return ((w & 0x7fff) > 0x7c00 ? 0 : w & 0xffff) | ((w >> 16 & 0x7fff) > 0x7c00 ? 0 : w & 0xffff0000u);
}
template <int D, bool PARTS>
__device__ __forceinline__ void kv4_make_ops(const char *stage, char *ops, const Kv4Part &part, const Kv4Scales &sc, int wave, int lane)
{
    typedef Kv4Stage<D> S;
    typedef Kv4Ops<D> O;
    constexpr int G = D / 32, KG = G / 2, VJ = D / 64;      // a wave's operands: KG groups of a tile's keys, VJ of the values
    const int q = lane >> 4;
    {
        const int i = wave >> 1, g0 = (wave & 1) * KG;
        uint32_t w[KG];
        lds_read(w, stage + S::k_read(i, lane) + g0 * 4);
#pragma unroll
        for (int g = 0; g < KG; g++) {
            Kv4Op o;
            kv4_widen<PARTS ? 8 : 0>(w[g], o.w);
            *(f16x8_t *)(ops + O::K + (i * G + g0 + g) * 1024 + lane * 16) = o.v;
        }
    }
    const _Float16 c = sc.big ? (_Float16)0.0625f : (_Float16)1.f;
    const f16x2_t c2 = {c, c}, c16 = c2 * f16x2_t{(_Float16)0.0625f, (_Float16)0.0625f};
    const bool all = part.all();
    {
        const int j0 = wave * VJ, g = j0 >> 1, h = j0 >> 2, shift = (j0 & 2) * 4;
        uint32_t w[4], sw[4], mw[4];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            uint32_t x[2], y[2], z[2] = {0, 0};
            lds_read(x, stage + S::v_read(i, lane) + h * 8);
            lds_read(y, stage + S::table(i, 2) + (q * G + g) * 8);
            if (!PARTS) lds_read(z, stage + S::table(i, 3) + (q * G + g) * 8);
#pragma unroll
            for (int a = 0; a < 2; a++) { w[2 * i + a] = x[a] >> shift; sw[2 * i + a] = y[a]; mw[2 * i + a] = z[a]; }
        }
        if (!all)
#pragma unroll
            for (int a = 0; a < 4; a++) {
                const uint32_t mask = kv4_pair_mask(4 * q + 2 * (a & 1), part.end(a >> 1));
                sw[a] &= mask; mw[a] &= mask;
            }
        if (sc.nan)
#pragma unroll
            for (int a = 0; a < 4; a++) sw[a] = kv4_nan_to_zero(sw[a]);
        f16x2_t hi[4], lo[4];
#pragma unroll
        for (int a = 0; a < 4; a++) {
            if (PARTS) {
                hi[a] = __builtin_bit_cast(f16x2_t, sw[a] & 0xfff0fff0u);
                lo[a] = __builtin_bit_cast(f16x2_t, sw[a]) - hi[a];
            } else {
                hi[a] = __builtin_bit_cast(f16x2_t, sw[a]);
                lo[a] = __builtin_bit_cast(f16x2_t, mw[a]) * c2;
            }
        }
        auto store = [&](int j, const f16x2_t (&n)[4]) {
            Kv4Op x, y;
#pragma unroll
            for (int a = 0; a < 4; a++) {
                x.w[a] = __builtin_bit_cast(uint32_t, PARTS ? n[a] * hi[a] : n[a] * hi[a] + lo[a]);
                y.w[a] = __builtin_bit_cast(uint32_t, n[a] * lo[a]);
            }
            *(f16x8_t *)(ops + O::VHI + j * 1024 + lane * 16) = x.v;
            if (PARTS) *(f16x8_t *)(ops + O::VLO + j * 1024 + lane * 16) = y.v;
        };
        f16x2_t n[4];
        if (VJ == 2 || (wave & 1) == 0) {
#pragma unroll
            for (int a = 0; a < 4; a++) n[a] = and_or(w[a], 0x000f000fu, 0x64006400u) * c2 - c2 * f16x2_t{(_Float16)(PARTS ? 1032 : 1024), (_Float16)(PARTS ? 1032 : 1024)};
            store(j0, n);
        }
        if (VJ == 2 || (wave & 1) == 1) {
#pragma unroll
            for (int a = 0; a < 4; a++) n[a] = and_or(w[a], 0x00f000f0u, 0x64006400u) * c16 - c2 * f16x2_t{(_Float16)(PARTS ? 72 : 64), (_Float16)(PARTS ? 72 : 64)};
            store(j0 + VJ - 1, n);
        }
    }
    if (PARTS && wave == 3) {                   // minima of the values: rows are groups, first parts, then the second ones
        const int g = lane & (G - 1), row = lane & 15;
        Kv4Op o;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            uint32_t x[2], y[2];
            lds_read(x, stage + S::table(i, 3) + (q * G + g) * 8);
            lds_read(y, stage + S::table(i, 2) + (q * G + g) * 8);
#pragma unroll
            for (int a = 0; a < 2; a++) {
                if (!all) {
                    const uint32_t mask = kv4_pair_mask(4 * q + 2 * a, part.end(i));
                    x[a] &= mask; y[a] &= mask;
                }
                if (sc.nan) y[a] = kv4_nan_to_zero(y[a]);
                uint32_t hi, lo;
                kv4_split(fmaf(half_of(y[a], 0), 8.f, half_of(x[a], 0)) * (float)c, fmaf(half_of(y[a], 1), 8.f, half_of(x[a], 1)) * (float)c, hi, lo);
                o.w[2 * i + a] = row < G ? hi : row < 2 * G ? lo : 0;
            }
        }
        *(f16x8_t *)(ops + O::VM + lane * 16) = o.v;
    }
    if (PARTS && wave < 2) {                    // minima of tile `wave`'s keys: first parts against both of the sums' (lane group 0), second against the first (1)
        const int tok = lane & 15;
        uint32_t km[G / 2], hi[2] = {0, 0}, lo[2] = {0, 0};
        lds_read(km, stage + S::table(wave, 1) + tok * 2 * G);
#pragma unroll
        for (int g = 0; g < G; g += 2) {
            const char *ks = stage + S::table(wave, 0) + ((tok >> 2) * G + g) * 8 + (tok & 3) * 2;
            kv4_split(fmaf((float)*(const _Float16 *)ks, 8.f, half_of(km[g / 2], 0)), fmaf((float)*(const _Float16 *)(ks + 8), 8.f, half_of(km[g / 2], 1)),
                      hi[g / 2], lo[g / 2]);
        }
        Kv4Op o;
#pragma unroll
        for (int g = 0; g < 2; g++) {
            o.w[g] = q == 0 ? hi[g] : q == 1 ? lo[g] : 0;
            o.w[2 + g] = q == 0 ? hi[g] : 0;
        }
        *(f16x8_t *)(ops + O::KM + wave * 1024 + lane * 16) = o.v;
    }
}

template <typename T, int D, int NC>
__global__ __launch_bounds__(256, 2) void kv4_attend_many_kernel(const Kv4Attn a)
{
    constexpr int G = D / 32, DT = D / 16;
    constexpr bool LO = sizeof(T) == 4, PARTS = !std::is_same<T, __bf16>::value;      // LO: fp32 rows, the queries' second part, and the product of both second parts
    typedef Kv4Stage<D> S;
    typedef Kv4Ops<D> O;
    __shared__ __align__(16) char raw[3 * S::BYTES], ops[2 * O::bytes(PARTS)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, h = blockIdx.y, chunk = blockIdx.z;
    const Kv4Cols k = kv4_columns<64 * NC>(a, (int)gridDim.x - 1 - (int)blockIdx.x);       // (late rows, which see most, first)
    if (k.s < 0) return;
    const int len = kv4_len(a.c, k.s), c0 = k.c0 + wave * 16 * NC, P = 1 << a.c.logT;
    int lim[NC];
    Kv4Column col[NC];
#pragma unroll
    for (int n = 0; n < NC; n++) {
        col[n] = kv4_column(a, k, h, c0 + 16 * n + (lane & 15), len);
        lim[n] = col[n].lim;
    }
    // what the wave's first and last column see, and the workgroup's last (later columns see no less)
    const int least = c0 < k.n ? kv4_row_lim(a, k, c0, len) : 0, most = c0 < k.n ? kv4_row_lim(a, k, min(c0 + 16 * NC, k.n) - 1, len) : 0;
    const int t0 = chunk * a.chunk, t1 = min(kv4_row_lim(a, k, min(k.c0 + 64 * NC, k.n) - 1, len), t0 + a.chunk);
    if (t0 >= t1 && chunk > 0) return;
    const uint32_t lds = lds_address(raw);
    int here = 0;                               // two bits a step: this one's lowest, then the next two's
    auto fetch = [&](int slot, int ahead, int t) {
        const Kv4Step st = kv4_step<D>(a.c, k.s, h, t, t1);
        here |= (st.here[0] | st.here[1] << 1) << (2 * ahead);
#pragma unroll
        for (int n = 0; n < S::LOADS; n++)
            if ((n & 3) == wave) S::load(n, st.blk[0], st.t[0], st.blk[1], st.t[1], P, lds + slot * S::BYTES, lane);
    };
    if (t0 < t1) fetch(0, 0, t0);
    if (t0 + 32 < t1) fetch(1, 1, t0 + 32);
    Kv4Query<D, LO> x[NC];
#pragma unroll
    for (int n = 0; n < NC; n++) {
        const Kv4Column col = kv4_column(a, k, h, c0 + 16 * n + (lane & 15), len);
        x[n].template load<PARTS>((const T *)a.q + (size_t)col.row * a.q_stride + (size_t)col.head * D, c0 + 16 * n + (lane & 15) < k.n,
                  kv4_aligned<T>(a.q, a.q_stride, 8), a.scale, q);
    }
    f32x4_t o[NC][DT], om[NC];
    float m[NC], l[NC];
#pragma unroll
    for (int n = 0; n < NC; n++) {
#pragma unroll
        for (int j = 0; j < DT; j++) o[n][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        om[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m[n] = -INFINITY; l[n] = 0.f;
    }
    loads_left<0>();
    __syncthreads();
    Kv4Scales sc = {false, false}, sc_next = sc;
    if (t0 < t1) {
        const Kv4Part part = {t1 - t0, here & 3};
        sc = kv4_scales<D>(raw, part, lane);
        kv4_make_ops<D, PARTS>(raw, ops, part, sc, wave, lane);
    }
    int slot = 0, buf = 0;
    for (int t = t0; t < t1; t += 32) {
        // here: this step's operands are made, the next one's numbers are in LDS, and all are done with what stood in the third place
        lds_reads_done();
        __syncthreads();
        const int next = slot == 2 ? 0 : slot + 1;
        if (t + 64 < t1) fetch(next == 2 ? 0 : next + 1, 2, t + 64);
        if (t + 32 < t1) {
            const Kv4Part part = {t1 - t - 32, here >> 2 & 3};
            const char *stage = raw + next * S::BYTES;
            sc_next = kv4_scales<D>(stage, part, lane);
            kv4_make_ops<D, PARTS>(stage, ops + (buf ^ 1) * O::bytes(PARTS), part, sc_next, wave, lane);
        }
        if (t < most) {
            const char *stage = raw + slot * S::BYTES, *op = ops + buf * O::bytes(PARTS);
            const Kv4Part part = {t1 - t, here & 3};
            const bool full = t + 32 <= least && part.all();
            f32x4_t z[2][NC];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint32_t ks[2 * G];
                lds_read(ks, stage + S::table(i, 0) + q * 8 * G);
                Kv4Op mm;
                if (PARTS) mm.v = *(const f16x8_t *)(op + O::KM + i * 1024 + lane * 16);
                else {
                    uint32_t km[G / 2];
                    lds_read(km, stage + S::table(i, 1) + (lane & 15) * 2 * G);
                    mm.w[0] = mm.w[2] = km[0];
                    mm.w[1] = mm.w[3] = G == 4 ? km[G / 2 - 1] : 0;
                }
                const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int n = 0; n < NC; n++) z[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(mm.v, x[n].sum.v, zero, 0, 0, 0);
#pragma unroll
                for (int g = 0; g < G; g++) {
                    const f16x8_t kk = *(const f16x8_t *)(op + O::K + (i * G + g) * 1024 + lane * 16);
#pragma unroll
                    for (int n = 0; n < NC; n++) {
                        f32x4_t d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, x[n].hi[g].v, zero, 0, 0, 0);
                        if (LO) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, x[n].lo[LO ? g : 0].v, d, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 4; j++) z[i][n][j] = fmaf(half_of(ks[2 * g + (j >> 1)], j & 1), d[j], z[i][n][j]);
                    }
                }
            }
            KV4_PART;
            Kv4Op hi[NC], lo[NC];
#pragma unroll
            for (int n = 0; n < NC; n++) {
                float y[8], mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; j++) y[j] = z[j >> 2][n][j & 3];
                if (!full)
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const int tok = 4 * q + (j & 3);
                        y[j] = tok < part.end(j >> 2) && t + 16 * (j >> 2) + tok < lim[n] ? y[j] : -INFINITY;
                    }
#pragma unroll
                for (int j = 0; j < 8; j++) mx = fmaxf(mx, y[j]);
                mx = quads_max(mx * x[n].f);
                if (__any(mx > m[n])) {
                    const float m_new = fmaxf(m[n], mx), alpha = __builtin_amdgcn_exp2f(m[n] - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
                    for (int j = 0; j < DT; j++) o[n][j] *= alpha;
                    om[n] *= alpha;
                    l[n] *= alpha;
                    m[n] = m_new;
                }
                const float ref = (m[n] == -INFINITY ? 0.f : m[n]) - a.shift - (sc.big ? 4.f : 0.f);
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; j++) p[j] = __builtin_amdgcn_exp2f(fmaf(y[j], x[n].f, -ref));
                const float sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                l[n] = fmaf(sum, sc.big ? 0.0625f : 1.f, l[n]);
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    if (PARTS) kv4_split(p[j], p[j + 1], hi[n].w[j >> 1], lo[n].w[j >> 1]);
                    else hi[n].w[j >> 1] = kv4_halves(p[j], p[j + 1]);
                }
            }
            KV4_PART;
            if (PARTS) {
                const f16x8_t vm = *(const f16x8_t *)(op + O::VM + lane * 16);
#pragma unroll
                for (int n = 0; n < NC; n++) {
                    om[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vm, hi[n].v, om[n], 0, 0, 0);
                    om[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vm, lo[n].v, om[n], 0, 0, 0);
                }
            }
#pragma unroll
            for (int j = 0; j < DT; j++) {
                const f16x8_t vh = *(const f16x8_t *)(op + O::VHI + j * 1024 + lane * 16);
#pragma unroll
                for (int n = 0; n < NC; n++) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, hi[n].v, o[n][j], 0, 0, 0);
                if (!PARTS) continue;
                const f16x8_t vl = *(const f16x8_t *)(op + O::VLO + j * 1024 + lane * 16);
#pragma unroll
                for (int n = 0; n < NC; n++) {
                    o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, lo[n].v, o[n][j], 0, 0, 0);
                    o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, hi[n].v, o[n][j], 0, 0, 0);
                    if (LO) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, lo[n].v, o[n][j], 0, 0, 0);
                }
            }
            if (sc.nan) {                       // a column that sees a group that is not a number has NaN there
#pragma unroll
                for (int n = 0; n < NC; n++)
#pragma unroll
                    for (int g = 0; g < G; g++) {
                        float seen = 0.f;
#pragma nounroll
                        for (int j = 0; j < 8; j++) {
                            const bool see = 4 * q + (j & 3) < part.end(j >> 2) && t + 16 * (j >> 2) + 4 * q + (j & 3) < lim[n];
                            const uint32_t w = *(const uint16_t *)(stage + S::table(j >> 2, 2) + (q * G + g) * 8 + (j & 3) * 2);
                            if (see && (w & 0x7fff) > 0x7c00) seen = 1.f;
                        }
                        if (quads_max(seen) > 0.f) om[n][g] = __builtin_nanf("");
                    }
            }
        }
        loads_left<0>();
        here >>= 2;
        sc = sc_next;
        slot = next;
        buf ^= 1;
    }
    const bool aligned = kv4_aligned<T>(a.out, a.out_stride, 4);
#pragma unroll
    for (int n = 0; n < NC; n++) {
        const float total = quads_sum(l[n]);
        // the groups' minima: first parts in the lanes of rows 0 .. G - 1, second in those of rows G .. 2 G - 1
#pragma unroll
        for (int g = 0; g < G; g++) {
            float v = __shfl(om[n][g], lane & 15);
            v += G == 4 ? __shfl(om[n][g], 16 + (lane & 15)) : __shfl(om[n][(g + 2) & 3], lane & 15);
#pragma unroll
            for (int j = 2 * g; j < 2 * g + 2; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) o[n][j][i] += v;
        }
        if (c0 + 16 * n + (lane & 15) >= k.n) continue;
        const Kv4Column col = kv4_column(a, k, h, c0 + 16 * n + (lane & 15), len);
        if (a.n_chunks > 1) {
            const size_t at = ((size_t)col.row * a.heads + col.head) * a.n_chunks + chunk;
#pragma unroll
            for (int j = 0; j < DT; j++) *(f32x4_t *)(a.part + at * D + 16 * j + 4 * q) = o[n][j];
            if (q == 0) a.part_ml[at] = float2{m[n], total};
        } else {
            T *out = (T *)a.out + (size_t)col.row * a.out_stride + (size_t)col.head * D;
#pragma unroll
            for (int j = 0; j < DT; j++) {
                f32x4_t y;
#pragma unroll
                for (int i = 0; i < 4; i++) y[i] = total == 0.f ? 0.f : o[n][j][i] / total;
                kv4_store4(out + 16 * j + 4 * q, aligned, y);
            }
            if (q == 0) a.lse[(size_t)col.row * a.heads + col.head] = total == 0.f ? -INFINITY : m[n] - a.shift + __builtin_amdgcn_logf(total);
        }
    }
}

// The chunks of a row that were written: those up to the last token that it sees (its block's other columns may see more).
__device__ __forceinline__ int kv4_row_chunks(const Kv4Attn &a, int lim) { return max(1, (lim + a.chunk - 1) / a.chunk); }

// Joins the chunks of a row and head, a workgroup each: wave w takes chunks w, w + 4, .., lane j of it the reference and sum of the j-th.
// A launch's latency: 3 us for 4 chunks of 32 heads, 4.8 for 16.
template <typename T, int D> __device__ __forceinline__ void kv4_join(const Kv4Attn &a, int item, float *lds)
{
    float (*os)[D] = (float (*)[D])lds, *ms = lds + 4 * D, *ls = ms + 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = item / a.heads, hq = item % a.heads;
    const Kv4Row row = kv4_row(a.c, a.row_start, r);
    if (row.s < 0) return;
    const int n = kv4_row_chunks(a, max(0, min(row.pos + 1, a.max_len))), mine = (n - wave + 3) / 4;
    const float2 *ml = a.part_ml + (size_t)item * a.n_chunks;
    const float *p = a.part + ((size_t)item * a.n_chunks + wave) * D + lane;
    const float2 c = lane < mine ? ml[wave + 4 * lane] : float2{-INFINITY, 0.f};
    float m = wave_max(c.x);
    if (lane == 0) ms[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
    const float f = __builtin_amdgcn_exp2f(c.x - (m == -INFINITY ? 0.f : m));
    const float l = wave_sum(f * c.y);
    float o[D / 64] = {};
#pragma unroll 8
    for (int j = 0; j < mine; j++) {
        const float fj = lane_value(f, j);
#pragma unroll
        for (int e = 0; e < D / 64; e++) o[e] = fmaf(fj, p[(size_t)j * 4 * D + 64 * e], o[e]);
    }
    if (lane == 0) ls[wave] = l;
#pragma unroll
    for (int e = 0; e < D / 64; e++) os[wave][lane + 64 * e] = o[e];
    __syncthreads();
    const float total = (ls[0] + ls[1]) + (ls[2] + ls[3]);
    if (threadIdx.x < D) {
        const float v = (os[0][threadIdx.x] + os[1][threadIdx.x]) + (os[2][threadIdx.x] + os[3][threadIdx.x]);
        ((T *)a.out)[(size_t)r * a.out_stride + (size_t)hq * D + threadIdx.x] = (T)(total == 0.f ? 0.f : v / total);
    }
}
template <typename T, int D> __global__ __launch_bounds__(256) void kv4_join_kernel(const Kv4Attn a)
{
    __shared__ float lds[4 * D + 8];
    kv4_join<T, D>(a, blockIdx.x, lds);
}

// One tile of 16 columns in LDS, for all waves of a workgroup.
template <int D, bool LO> struct Kv4Tile {
    f16x8_t hi[D / 32][64], lo[LO ? D / 32 : 1][64], sum[64];
    float f[16], lse[16];
    int lim[16];
};
// base-2 logarithm of a column's sum: from its chunks, where there are several
__device__ __forceinline__ float kv4_lse(const Kv4Attn &a, size_t item, int lim, int q)
{
    if (a.n_chunks == 1) return a.lse[item];
    const int n = kv4_row_chunks(a, lim);
    const float2 *ml = a.part_ml + item * a.n_chunks;
    float m = -INFINITY, l = 0.f;
#pragma unroll 8
    for (int i = q; i < n; i += 4) m = fmaxf(m, ml[i].x);
    m = quads_max(m);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 8
    for (int i = q; i < n; i += 4) l = fmaf(__builtin_amdgcn_exp2f(ml[i].x - ref), ml[i].y, l);
    l = quads_sum(l);
    return l == 0.f ? -INFINITY : m - a.shift + __builtin_amdgcn_logf(l);
}

// What follows the chunks of a call with weights, in one launch: workgroups below n_join join a row and head (none where there is one chunk);
// the others take 128 tokens of a sequence and cache head, 32 a wave, and go over all columns that see them:
//     w_out[t] = w_in[t] + sum over the columns of 2^(z - lse), the scores those of the attention.
// Four tiles of columns at a time are made ready in LDS, one by each wave.  Bound by that preparation where there are few columns (7 rows of 32
// heads, 4103 tokens 13 to 15 us; several blocks of tokens over one preparation gain a twentieth there and lose one in a hundred with prompts) and
// by exponentials and their sums with prompts (777 and 131 rows of 40 heads 50 us).
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void kv4_weights_kernel(const Kv4Attn a, int n_join, int token_blocks)
{
    constexpr int G = D / 32;
    constexpr bool LO = sizeof(T) == 4;
    __shared__ __align__(16) Kv4Tile<D, LO> tiles[4];
    if ((int)blockIdx.x < n_join) {
        kv4_join<T, D>(a, blockIdx.x, (float *)tiles);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, P = 1 << a.c.logT;
    const int b = blockIdx.x - n_join, hs = b / token_blocks, h = hs % a.c.H, s = hs / a.c.H, first = (b % token_blocks) * 128, t0 = first + 32 * wave;
    const int len = kv4_len(a.c, s), n = min(len, a.max_len);
    if (first >= n) return;
    Kv4Cols k;
    k.s = s; k.c0 = 0;
    k.r0 = min(max(a.row_start[s], 0), a.n_rows); k.end = a.row_start[s + 1];
    k.n = (min(max(k.end, k.r0), a.n_rows) - k.r0) * a.group;
    const Kv4Step st = kv4_step<D>(a.c, s, h, t0, n);
    Kv4Keys<D> keys[2];
    f16x8_t kk[2][G];
#pragma unroll
    for (int i = 0; i < 2; i++) keys[i].load_page(st.blk[i], P, st.t[i], lane);
    const size_t at = ((size_t)s * a.c.H + h) * ((size_t)a.c.max_pages << a.c.logT);
    float old = 0.f;
    const int mine = t0 + 16 * (lane >> 2 & 1) + 4 * q + (lane & 3);        // the token whose weight this lane writes, lane % 16 below 8
    const bool writes = (lane & 8) == 0 && mine < n;
    if (a.w_in && writes) old = a.w_in[at + mine];
#pragma unroll
    for (int i = 0; i < 2; i++) keys[i].widen(kk[i]);
    float sum[8] = {};
    // columns in front of the first that sees the workgroup's first token see none of its tokens
    const int row = first - (len - k.end + k.r0);
    for (int c0 = (row > 0 ? min(row, k.n) * a.group : 0) & ~15; c0 < k.n; c0 += 64) {
        __syncthreads();                        // (the tiles before these have been read)
        if (c0 + 16 * wave < k.n) {
            const int cc = c0 + 16 * wave + (lane & 15);
            const Kv4Column col = kv4_column(a, k, h, cc, len);
            Kv4Query<D, LO> x;
            x.load((const T *)a.q + (size_t)col.row * a.q_stride + (size_t)col.head * D, cc < k.n, kv4_aligned<T>(a.q, a.q_stride, 8), a.scale, q);
            const float lse = cc < k.n ? kv4_lse(a, (size_t)col.row * a.heads + col.head, col.lim, q) : 0.f;
            Kv4Tile<D, LO> &tile = tiles[wave];
#pragma unroll
            for (int g = 0; g < G; g++) {
                tile.hi[g][lane] = x.hi[g].v;
                if (LO) tile.lo[LO ? g : 0][lane] = x.lo[LO ? g : 0].v;
            }
            tile.sum[lane] = x.sum.v;
            if (q == 0) { tile.f[lane] = x.f; tile.lse[lane] = lse; tile.lim[lane] = col.lim; }
        }
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < 4 && c0 + 16 * i < k.n; i++) {
            const Kv4Tile<D, LO> &tile = tiles[i];
            Kv4Query<D, LO> x;
#pragma unroll
            for (int g = 0; g < G; g++) {
                x.hi[g].v = tile.hi[g][lane];
                if (LO) x.lo[LO ? g : 0].v = tile.lo[LO ? g : 0][lane];
            }
            x.sum.v = tile.sum[lane];
            const float f = tile.f[lane & 15], lse = tile.lse[lane & 15];
            const int lim = tile.lim[lane & 15];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const f32x4_t z = keys[u].scores(kk[u], x);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(z[j], f, -lse));
                    sum[4 * u + j] += st.here[u] && t0 + 16 * u + 4 * q + j < lim ? p : 0.f;
                }
            }
        }
    }
    // over the 16 columns of a tile; lane l % 16 = j keeps the sum of token j
    float total = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float v = row_sum(sum[j]);
        total = (lane & 7) == j ? v : total;
    }
    if (writes) a.w_out[at + mine] = old + total;
}

// ---- eviction -----------------------------------------------------------------------------------

// Order of the weights as unsigned numbers: NaN above all, -0 = +0.
__device__ __forceinline__ uint32_t kv4_key(float w)
{
    uint32_t b = __float_as_uint(w);
    if (w != w) return 0xffffffffu;
    if (b == 0x80000000u) b = 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Kv4Evict {
    Kv4View src, dst;
    int keep, first, recent;
    const float *w_in;
    float *w_out;
    int *kept;
};

// Which tokens of a sequence and head stay: radix selection of the need-th largest weight (digits of 11, 11 and 10 bits), then the tokens
// in order with their ranks.  One workgroup per sequence and head.  A thread takes consecutive tokens, up to 32 of a segment of 32768, so
// that one scan over the workgroup ranks a whole segment; the weights come from the L2 again in every pass.  Weights share few exponents,
// so the histogram is held eight times over (lane % 8) against conflicts.  4096 of 32 heads: 16 us; with digits of 8 bits, one histogram
// and a serial search of it 36.
constexpr int KV4_SEG = 32, KV4_COPIES = 8, KV4_BINS = 2048 + 8;      // (8: copies of a digit lie in different banks)
__device__ __forceinline__ int block_scan(int v, int *tmp, int &total)     // exclusive, 1024 threads; tmp [16]
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(x, o);
        if (lane >= o) x += u;
    }
    __syncthreads();                            // (tmp of an earlier scan has been read)
    if (lane == 63) tmp[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int t = tmp[i];
        before += i < wave ? t : 0;
        total += t;
    }
    return before + x - v;
}

__global__ __launch_bounds__(1024) void kv4_select_kernel(const Kv4Evict a)
{
    __shared__ int hist[KV4_COPIES * KV4_BINS], tmp[16], found[2];
    const int s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
    const size_t in_cap = (size_t)a.src.max_pages << a.src.logT, out_cap = (size_t)a.dst.max_pages << a.dst.logT;
    const float *w = a.w_in + ((size_t)s * a.src.H + h) * in_cap;       // (in_cap is a multiple of 16, so every row is 16-byte aligned if the first is)
    float *wo = a.w_out + ((size_t)s * a.src.H + h) * out_cap;
    int *kept = a.kept + ((size_t)s * a.src.H + h) * a.keep;
    const int n = kv4_len(a.src, s), m = min(n, a.keep);
    for (size_t i = m + tid; i < out_cap; i += 1024) wo[i] = 0.f;
    for (int i = m + tid; i < a.keep; i += 1024) kept[i] = -1;
    if (n <= a.keep) {
        for (int i = tid; i < n; i += 1024) { kept[i] = i; wo[i] = w[i]; }
        return;
    }
    const int lo = a.first, hi = n - a.recent, need = a.keep - a.first - a.recent;
    // tokens per thread and segment: a multiple of 4
    const int per = min(KV4_SEG, (n + 4095) / 4096 * 4), seg = per * 1024;
    const bool aligned = ((uintptr_t)a.w_in & 15) == 0;
    auto load4 = [&](int t, float (&x)[4]) {    // tokens t..t + 3, t a multiple of 4 below n (a row's memory goes on to a multiple of 16)
        if (aligned) {
            const float4 v = *(const float4 *)(w + t);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = w[t + e];
        }
    };
    uint32_t prefix = 0;
    int want = need;                            // of the candidates whose leading digits are prefix's
#pragma unroll
    for (int pass = 0; pass < 3; pass++) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass < 2 ? 11 : 10;
        if (!need) break;
        for (int i = tid; i < KV4_COPIES * KV4_BINS; i += 1024) hist[i] = 0;
        __syncthreads();
        for (int s0 = 0; s0 < n; s0 += seg) {
#pragma unroll
            for (int i = 0; i < KV4_SEG / 4; i++) {
                const int t = s0 + i * 4096 + tid * 4;          // (here the order does not matter: neighbouring lanes read neighbouring tokens)
                if (i * 4 >= per || t >= n) continue;
                float x[4];
                load4(t, x);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t k = kv4_key(x[e]);
                    if (t + e >= lo && t + e < hi && (pass == 0 || k >> (shift + bits) == prefix >> (shift + bits)))
                        atomicAdd(&hist[(k >> shift & ((1u << bits) - 1)) + (tid & (KV4_COPIES - 1)) * KV4_BINS], 1);
                }
            }
        }
        __syncthreads();
        // thread i looks at digits 2047 - 2 i and 2046 - 2 i: how many candidates lie above them
        int c[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            c[e] = 0;
#pragma unroll
            for (int j = 0; j < KV4_COPIES; j++) c[e] += hist[2047 - 2 * tid - e + j * KV4_BINS];
        }
        int total, above = block_scan(c[0] + c[1], tmp, total);
#pragma unroll
        for (int e = 0; e < 2; e++) {
            if (above < want && above + c[e] >= want) { found[0] = 2047 - 2 * tid - e; found[1] = want - above; }
            above += c[e];
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        want = found[1];
        __syncthreads();
    }
    // tokens above the threshold, and the first `want` that equal it
    int above = 0, equal = 0;
    for (int s0 = 0; s0 < n; s0 += seg) {
        const int t0 = s0 + tid * per;
        uint32_t up = 0, eq = 0;
#pragma unroll
        for (int i = 0; i < KV4_SEG / 4; i++) {
            const int t = t0 + 4 * i;
            if (i * 4 >= per || t >= n) continue;
            float x[4];
            load4(t, x);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint32_t k = kv4_key(x[e]);
                const bool in = t + e < n, forced = in && (t + e < lo || t + e >= hi), cand = in && !forced && need;
                up |= (uint32_t)(forced || (cand && k > prefix)) << (4 * i + e);
                eq |= (uint32_t)(cand && k == prefix) << (4 * i + e);
            }
        }
        int total_up, total_eq;
        const int before_up = block_scan(__popc(up), tmp, total_up), before_eq = block_scan(__popc(eq), tmp, total_eq);
        int pos = above + before_up + min(equal + before_eq, want), ties = equal + before_eq;
        for (uint32_t any = up | eq; any; any &= any - 1) {
            const int i = __builtin_ctz(any);
            if (eq >> i & 1) {
                if (ties >= want) continue;
                ties++;
            }
            kept[pos] = t0 + i; wo[pos] = w[t0 + i];
            pos++;
        }
        above += total_up; equal += total_eq;
    }
}

// The kept tokens' numbers, moved together.  Four tokens of the new page per 16 lanes: lane l carries piece l % 4 of the keys of token l / 4, the
// values' halfwords r = l of all four, and one number of each of the four tables of scales.  Bound by gathering the values two bytes at a time:
// 2048 of 4096 tokens, 32 heads (21 MB read and written) 21 us; the tables four tokens at a time instead: 22.
template <int D>
__global__ __launch_bounds__(256) void kv4_move_kernel(const Kv4Evict a)
{
    typedef Kv4<D> L;
    constexpr int G = L::G, VH = L::VH, KW = D / 32;        // words of a lane's piece of a token's keys
    const int s = blockIdx.z, h = blockIdx.y, li = threadIdx.x & 15, quad = blockIdx.x * 16 + (threadIdx.x >> 4);
    const int P = 1 << a.src.logT, Q = 1 << a.dst.logT, n = kv4_len(a.src, s), m = min(n, a.keep);
    if (quad * 4 >= m) return;
    char *dst = kv4_block<D>(a.dst, s, h, quad * 4);        // (quad * 4 < n_keep, which the page table reaches)
    if (!dst) return;
    const int *kept = a.kept + ((size_t)s * a.src.H + h) * a.keep + quad * 4;
    const int u = quad * 4 & (Q - 1), last = m - quad * 4;  // tokens of the quad that there are, if fewer than 4
    const char *src[4];
    int t[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int from = i < last ? kept[i] : 0;
        t[i] = from & (P - 1);
        src[i] = i < last ? kv4_block<D>(a.src, s, h, from) : nullptr;
    }
    // the lane's own token of the four
    const int mine = li >> 2, piece = li & 3;
    const char *ms = mine == 0 ? src[0] : mine == 1 ? src[1] : mine == 2 ? src[2] : src[3];
    const int mt = mine == 0 ? t[0] : mine == 1 ? t[1] : mine == 2 ? t[2] : t[3];
    uint32_t kw[KW] = {};
    uint16_t vw[VH][4] = {}, ks = 0, km = 0, vs = 0, vm = 0;
    if (ms) {
        __builtin_memcpy(kw, __builtin_assume_aligned(ms + mt * (D / 2) + piece * 4 * KW, 4 * KW), 4 * KW);
        if (piece < G) {
            ks = *(const uint16_t *)(ms + L::ks(P, mt, piece)); km = *(const uint16_t *)(ms + L::km(P, mt, piece));
            vs = *(const uint16_t *)(ms + L::vs(P, mt, piece)); vm = *(const uint16_t *)(ms + L::vm(P, mt, piece));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (src[i])
#pragma unroll
            for (int k = 0; k < VH; k++) vw[k][i] = *(const uint16_t *)(src[i] + L::v_half(P, t[i], li, k));
    if (mine < last) {
        __builtin_memcpy(__builtin_assume_aligned(dst + (u + mine) * (D / 2) + piece * 4 * KW, 4 * KW), kw, 4 * KW);
        if (piece < G) {
            *(uint16_t *)(dst + L::ks(Q, u + mine, piece)) = ks; *(uint16_t *)(dst + L::km(Q, u + mine, piece)) = km;
            *(uint16_t *)(dst + L::vs(Q, u + mine, piece)) = vs; *(uint16_t *)(dst + L::vm(Q, u + mine, piece)) = vm;
        }
    }
    if (last >= 4) __builtin_memcpy(__builtin_assume_aligned(dst + L::v_half(Q, u, li, 0), 8 * VH), vw, 8 * VH);
    else
        for (int i = 0; i < last; i++)
#pragma unroll
            for (int k = 0; k < VH; k++) *(uint16_t *)(dst + L::v_half(Q, u + i, li, k)) = vw[k][i];
}
