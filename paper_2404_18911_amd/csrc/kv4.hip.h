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

template <typename T> __device__ __forceinline__ float row_ld(const T *p) { return (float)*p; }

// The 16 levels of a group.  lo, hi: its least and largest component (clamped), bad: one of them is not finite.
struct Kv4Levels { float s, m; };
__device__ __forceinline__ Kv4Levels kv4_levels(float lo, float hi, bool bad)
{
    Kv4Levels l;
    l.m = bad ? 0.f : (float)(_Float16)lo;
    l.s = bad ? __builtin_nanf("") : (float)(_Float16)__fdiv_rn(__fsub_rn(hi, lo), 15.f);
    return l;
}
// n = clamp(rint((x - m) / s), 0, 15) of the exact quotient: the rounded one of fp32 errs next to a border, so its residual is checked in 64 bits
__device__ __forceinline__ uint32_t kv4_level(float x, const Kv4Levels &l)
{
    if (!(l.s > 0.f)) return 0;
    float n = fminf(fmaxf(rintf((x - l.m) / l.s), 0.f), 15.f);
    const double s = l.s, rest = fma(-(double)n, s, (double)x - (double)l.m) * 2.0;
    const bool odd = (int)n & 1;
    if (rest > s || (rest == s && odd)) n += 1.f;
    else if (rest < -s || (rest == -s && odd)) n -= 1.f;
    return (uint32_t)fminf(fmaxf(n, 0.f), 15.f);
}
__device__ __forceinline__ float kv4_clamp(float x) { return fminf(fmaxf(x, -65504.f), 65504.f); }
__device__ __forceinline__ bool kv4_bad(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// One row and head per D / 8 lanes, eight components each.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4View c, const T *k, long k_stride, const T *v, long v_stride, const int *row_start,
                                                         int n_rows)
{
    typedef Kv4<D> L;
    constexpr int LP = D / 8;
    const int li = threadIdx.x & (LP - 1), lane = threadIdx.x & 63;
    const size_t item = (size_t)blockIdx.x * (256 / LP) + threadIdx.x / LP;
    const int r = (int)(item / c.H), h = (int)(item % c.H), P = 1 << c.logT;
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
        float x[8], lo = INFINITY, hi = -INFINITY;
        bool bad = false;
        for (int e = 0; e < 8; e++) {
            x[e] = live ? row_ld(k + (size_t)r * k_stride + (size_t)h * D + 32 * g + 8 * q + e) : 0.f;
            bad |= kv4_bad(x[e]);
            x[e] = kv4_clamp(x[e]);
            lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]);
        }
        for (int o = 1; o < 4; o <<= 1) { lo = fminf(lo, __shfl_xor(lo, o)); hi = fmaxf(hi, __shfl_xor(hi, o)); }
        const Kv4Levels l = kv4_levels(lo, hi, (__ballot(bad) >> (lane & ~3)) & 15);
        uint32_t w = 0;
        for (int e = 0; e < 8; e++) w |= kv4_level(x[e], l) << (4 * e);
        if (live) {
            *(uint32_t *)(blk + L::k_word(P, t, q, g)) = w;
            if (q == 0) {
                *(_Float16 *)(blk + L::ks(P, t, g)) = (_Float16)l.s;
                *(_Float16 *)(blk + L::km(P, t, g)) = (_Float16)l.m;
            }
        }
    }
    // values: component 16 j + r, lane li has r = li (D = 128: j = 0..7) or r = li, li + 8 (D = 64: j = 0..3 each)
    float x[8];
    bool bad[8];
    for (int e = 0; e < 8; e++) {
        const int d = D == 128 ? 16 * e + li : 16 * (e & 3) + li + 8 * (e >> 2);
        x[e] = live ? row_ld(v + (size_t)r * v_stride + (size_t)h * D + d) : 0.f;
        bad[e] = kv4_bad(x[e]);
        x[e] = kv4_clamp(x[e]);
    }
    uint32_t w[2] = {0, 0};
    for (int g = 0; g < L::G; g++) {
        // the elements of group g: j = 2 g, 2 g + 1
        float lo = INFINITY, hi = -INFINITY;
        bool b = false;
        for (int e = 0; e < 8; e++) {
            if ((D == 128 ? e : e & 3) >> 1 != g) continue;
            lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]);
            b |= bad[e];
        }
        for (int o = 1; o < LP; o <<= 1) { lo = fminf(lo, __shfl_xor(lo, o)); hi = fmaxf(hi, __shfl_xor(hi, o)); }
        const Kv4Levels l = kv4_levels(lo, hi, (__ballot(b) >> (lane & ~(LP - 1))) & ((1ull << LP) - 1));
        for (int e = 0; e < 8; e++) {
            if ((D == 128 ? e : e & 3) >> 1 != g) continue;
            w[e >> 2] |= kv4_level(x[e], l) << (4 * (e & 3));
        }
        if (live && li == g) {
            *(_Float16 *)(blk + L::vs(P, t, g)) = (_Float16)l.s;
            *(_Float16 *)(blk + L::vm(P, t, g)) = (_Float16)l.m;
        }
    }
    if (live) {
        for (int i = 0; i < 2; i++)
            *(uint16_t *)(blk + (D == 128 ? L::v_half(P, t, li, i) : L::v_half(P, t, li + 8 * i, 0))) = (uint16_t)w[i];
    }
}

// Keys and values of the rows, widened.  A token without a page reads as zeros.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4View c, T *k, long k_stride, T *v, long v_stride, const int *row_start, int n_rows)
{
    typedef Kv4<D> L;
    constexpr int LP = D / 8;
    const int li = threadIdx.x & (LP - 1);
    const size_t item = (size_t)blockIdx.x * (256 / LP) + threadIdx.x / LP;
    const int r = (int)(item / c.H), h = (int)(item % c.H), P = 1 << c.logT;
    if (r >= n_rows) return;
    const Kv4Row row = kv4_row(c, row_start, r);
    if (row.s < 0 || row.pos < 0) return;
    const char *blk = kv4_block<D>(c, row.s, h, row.pos);
    const int t = row.pos & (P - 1);
    for (int e = 0; e < 8; e++) {
        const int d = 8 * li + e, g = d >> 5, j = d >> 4, rr = d & 15;
        float kx = 0.f, vx = 0.f;
        if (blk) {
            const uint32_t kw = *(const uint32_t *)(blk + L::k_word(P, t, (d & 31) >> 3, g)) >> (4 * (d & 7)) & 15;
            const uint32_t vw = *(const uint16_t *)(blk + L::v_half(P, t, rr, j >> 2)) >> (4 * (j & 3)) & 15;
            kx = fmaf((float)*(const _Float16 *)(blk + L::ks(P, t, g)), (float)kw, (float)*(const _Float16 *)(blk + L::km(P, t, g)));
            vx = fmaf((float)*(const _Float16 *)(blk + L::vs(P, t, g)), (float)vw, (float)*(const _Float16 *)(blk + L::vm(P, t, g)));
        }
        k[(size_t)r * k_stride + (size_t)h * D + d] = (T)kx;
        v[(size_t)r * v_stride + (size_t)h * D + d] = (T)vx;
    }
}

struct Kv4Attn {
    Kv4View c;
    const void *q;
    void *out;
    long q_stride, out_stride;
    const int *row_start;
    int n_rows, heads, max_len;
    float scale;
    const float *w_in;
    float *w_out, *lse;          // lse [row][head], base 2
};

// One row and head per workgroup, a token per thread.
template <typename T, int D>
__global__ __launch_bounds__(128) void kv4_attend_kernel(const Kv4Attn a)
{
    typedef Kv4<D> L;
    __shared__ float qs[D], ps[128], red[2];
    const int r = blockIdx.x, hq = blockIdx.y, h = hq / (a.heads / a.c.H), P = 1 << a.c.logT, tid = threadIdx.x;
    const Kv4Row row = kv4_row(a.c, a.row_start, r);
    if (row.s < 0) return;
    for (int d = tid; d < D; d += 128) qs[d] = row_ld((const T *)a.q + (size_t)r * a.q_stride + (size_t)hq * D + d) * (a.scale * 1.44269504f);
    __syncthreads();
    const int n = min(row.pos + 1, a.max_len);
    float mx = -INFINITY, l = 0.f, o = 0.f;
    for (int t0 = 0; t0 < n; t0 += 128) {
        const int t = t0 + tid;
        float sc = -INFINITY;
        const char *blk = t < n ? kv4_block<D>(a.c, row.s, h, t) : nullptr;
        if (blk) {
            const int tp = t & (P - 1);
            sc = 0.f;
            for (int d = 0; d < D; d++) {
                const int g = d >> 5;
                const uint32_t kw = *(const uint32_t *)(blk + L::k_word(P, tp, (d & 31) >> 3, g)) >> (4 * (d & 7)) & 15;
                sc = fmaf(qs[d], fmaf((float)*(const _Float16 *)(blk + L::ks(P, tp, g)), (float)kw, (float)*(const _Float16 *)(blk + L::km(P, tp, g))), sc);
            }
        }
        float m = sc;
        for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
        if ((tid & 63) == 0) red[tid >> 6] = m;
        __syncthreads();
        m = fmaxf(mx, fmaxf(red[0], red[1]));
        const float p = blk ? exp2f(sc - m) : 0.f;
        ps[tid] = p;
        __syncthreads();
        const float alpha = mx == -INFINITY ? 0.f : exp2f(mx - m);
        mx = m;
        o *= alpha; l *= alpha;
        for (int i = 0; i < 128 && t0 + i < n; i++) {
            l += ps[i];
            const char *b = kv4_block<D>(a.c, row.s, h, t0 + i);
            if (!b || tid >= D) continue;
            const int j = tid >> 4, tp = (t0 + i) & (P - 1);
            const uint32_t vw = *(const uint16_t *)(b + L::v_half(P, tp, tid & 15, j >> 2)) >> (4 * (j & 3)) & 15;
            o = fmaf(ps[i], fmaf((float)*(const _Float16 *)(b + L::vs(P, tp, tid >> 5)), (float)vw, (float)*(const _Float16 *)(b + L::vm(P, tp, tid >> 5))), o);
        }
        __syncthreads();
    }
    if (tid < D) ((T *)a.out)[(size_t)r * a.out_stride + (size_t)hq * D + tid] = (T)(l == 0.f ? 0.f : o / l);
    if (tid == 0) a.lse[(size_t)r * a.heads + hq] = l == 0.f ? -INFINITY : mx + log2f(l);
}

// w_out[s][h][t] = w_in + the probabilities of token t, summed over the rows and the query heads of head h.  A thread per token.
template <typename T, int D>
__global__ __launch_bounds__(128) void kv4_weights_kernel(const Kv4Attn a)
{
    typedef Kv4<D> L;
    __shared__ float qs[D];
    const int s = blockIdx.z, h = blockIdx.y, t = blockIdx.x * 128 + threadIdx.x, P = 1 << a.c.logT, g = a.heads / a.c.H;
    const int len = kv4_len(a.c, s), n = min(len, a.max_len);
    if ((int)blockIdx.x * 128 >= n) return;
    const char *blk = t < n ? kv4_block<D>(a.c, s, h, t) : nullptr;
    const size_t at = ((size_t)s * a.c.H + h) * ((size_t)a.c.max_pages << a.c.logT) + t;
    float sum = 0.f;
    const int r0 = max(a.row_start[s], 0), r1 = min(a.row_start[s + 1], a.n_rows);
    for (int r = r0; r < r1; r++) {
        for (int hq = h * g; hq < h * g + g; hq++) {
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += 128) qs[d] = row_ld((const T *)a.q + (size_t)r * a.q_stride + (size_t)hq * D + d) * (a.scale * 1.44269504f);
            __syncthreads();
            if (!blk || t > len - a.row_start[s + 1] + r) continue;
            float sc = 0.f;
            const int tp = t & (P - 1);
            for (int d = 0; d < D; d++) {
                const int gr = d >> 5;
                const uint32_t kw = *(const uint32_t *)(blk + L::k_word(P, tp, (d & 31) >> 3, gr)) >> (4 * (d & 7)) & 15;
                sc = fmaf(qs[d], fmaf((float)*(const _Float16 *)(blk + L::ks(P, tp, gr)), (float)kw, (float)*(const _Float16 *)(blk + L::km(P, tp, gr))), sc);
            }
            sum += exp2f(sc - a.lse[(size_t)r * a.heads + hq]);
        }
    }
    if (t < n) a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + sum;
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

// Which tokens of a sequence and head stay: radix selection of the need-th largest weight (four digits of 8 bits), then the tokens
// in order with their ranks.  One workgroup per sequence and head.
__global__ __launch_bounds__(1024) void kv4_select_kernel(const Kv4Evict a)
{
    __shared__ int hist[256], scan[16], digit, left;
    const int s = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const size_t in_cap = (size_t)a.src.max_pages << a.src.logT, out_cap = (size_t)a.dst.max_pages << a.dst.logT;
    const float *w = a.w_in + ((size_t)s * a.src.H + h) * in_cap;
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
    uint32_t prefix = 0;
    int want = need;                            // of the candidates whose leading digits are prefix's
    for (int shift = 24; shift >= 0 && need; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += 1024) {
            const uint32_t k = kv4_key(w[i]);
            if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[k >> shift & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int c = 0, d = 255;
            while (d > 0 && c + hist[d] < want) c += hist[d--];
            digit = d; left = want - c;
        }
        __syncthreads();
        prefix |= (uint32_t)digit << shift;
        want = left;
        __syncthreads();
    }
    // tokens above the threshold, and the first `want` that equal it
    int above = 0, equal = 0;
    for (int t0 = 0; t0 < n; t0 += 1024) {
        const int t = t0 + tid;
        int f = 0;                              // 1: stays, 0x10000: equals the threshold
        if (t < n) {
            if (t < lo || t >= hi) f = 1;
            else if (need) {
                const uint32_t k = kv4_key(w[t]);
                f = k > prefix ? 1 : k == prefix ? 0x10000 : 0;
            }
        }
        int v = f;
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(v, o);
            if (lane >= o) v += u;
        }
        if (lane == 63) scan[wave] = v;
        __syncthreads();
        int before = 0, total = 0;
        for (int i = 0; i < 16; i++) {
            if (i < wave) before += scan[i];
            total += scan[i];
        }
        __syncthreads();
        const int ex = before + v - f, e = equal + (ex >> 16), pos = above + (ex & 0xffff) + min(e, want);
        if (f == 1 || (f && e < want)) { kept[pos] = t; wo[pos] = w[t]; }
        above += total & 0xffff; equal += total >> 16;
    }
}

// The kept tokens' numbers, moved together.  Four tokens of the new page per 16 lanes.
template <int D>
__global__ __launch_bounds__(256) void kv4_move_kernel(const Kv4Evict a)
{
    typedef Kv4<D> L;
    const int s = blockIdx.z, h = blockIdx.y, li = threadIdx.x & 15, quad = blockIdx.x * 16 + (threadIdx.x >> 4);
    const int P = 1 << a.src.logT, Q = 1 << a.dst.logT, n = kv4_len(a.src, s), m = min(n, a.keep);
    if (quad * 4 >= m) return;
    char *dst = (quad * 4 >> a.dst.logT) < a.dst.max_pages ? kv4_block<D>(a.dst, s, h, quad * 4) : nullptr;
    if (!dst) return;
    const int *kept = a.kept + ((size_t)s * a.src.H + h) * a.keep + quad * 4;
    for (int i = 0; i < 4 && quad * 4 + i < m; i++) {
        const int from = kept[i], t = from & (P - 1), u = (quad * 4 + i) & (Q - 1);
        const char *src = kv4_block<D>(a.src, s, h, from);
        for (int w = li; w < D / 8; w += 16) *(uint32_t *)(dst + u * (D / 2) + 4 * w) = src ? *(const uint32_t *)(src + t * (D / 2) + 4 * w) : 0;
        for (int k = 0; k < L::VH; k++)
            *(uint16_t *)(dst + L::v_half(Q, u, li, k)) = src ? *(const uint16_t *)(src + L::v_half(P, t, li, k)) : 0;
        if (li < L::G) {
            *(uint16_t *)(dst + L::ks(Q, u, li)) = src ? *(const uint16_t *)(src + L::ks(P, t, li)) : 0;
            *(uint16_t *)(dst + L::km(Q, u, li)) = src ? *(const uint16_t *)(src + L::km(P, t, li)) : 0;
            *(uint16_t *)(dst + L::vs(Q, u, li)) = src ? *(const uint16_t *)(src + L::vs(P, t, li)) : 0;
            *(uint16_t *)(dst + L::vm(Q, u, li)) = src ? *(const uint16_t *)(src + L::vm(P, t, li)) : 0;
        }
    }
}
