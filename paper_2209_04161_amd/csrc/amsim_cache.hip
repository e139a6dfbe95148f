// amsim_cache.hip -- a paged cache of keys and values held in 8 bits with a scale for each page and head:
// the append that fills it and the attention that reads it.
//
// Layout: keys [page][head][token][d], values [page][head][d][token] (each page's values transposed, so
// that the lanes of the second product read runs of tokens), scales [page][head].
#include <type_traits>

#include "amsim_q8.h"

namespace {

using namespace amsim_q8;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// What the calls take of a batch: the page table, each sequence's length with its new tokens, and where its
// new tokens lie.  Numbers that do not fit the tensors are cut to what does, so that a wrong table or
// length gives wrong results but no access outside them.
struct Seqs {
    const int *table, *lengths, *starts;
    int64_t ld_table;
    int batch, max_new, total_new, n_pages, page, shift;  // page = 1 << shift
    int64_t max_len;
};

struct Seq {
    int len, nq, start;
};

__device__ __forceinline__ Seq sequence(const Seqs &s, int b)
{
    const int64_t most = s.max_len < s.ld_table * s.page ? s.max_len : s.ld_table * s.page;
    const int64_t len = s.lengths[b];
    Seq r;
    r.len = int(len < 0 ? 0 : (len > most ? most : len));
    const int lo = s.starts[b], hi = s.starts[b + 1];
    r.start = lo < 0 ? 0 : (lo > s.total_new ? s.total_new : lo);
    const int end = hi < r.start ? r.start : (hi > s.total_new ? s.total_new : hi);
    r.nq = end - r.start < s.max_new ? end - r.start : s.max_new;
    return r;
}

// ------------------------------------------------------------------ append ---------------

struct AppendArgs {
    Seqs s;
    const void *src[2];
    int64_t tok[2], head[2];
    int8_t *pool[2];
    float *scale[2];
    int heads, d, touched;
    unsigned first;  // the launch's first workgroup
};

// One workgroup to a page that gets new tokens, a head, and keys or values: the new tokens' largest
// magnitude, then the page's bytes.  Keys by 16 elements of a token; values, which the page holds transposed, by 8
// elements of 4 tokens, neighbouring lanes taking neighbouring tokens, so that 64 tokens' bytes of one element
// are written together (gathered one element at a time they took twice as long: 35 us against 18 for
// 1500 tokens of 5 sequences).  Bound by memory for long runs of tokens; for single ones by the chain of
// dependent reads (length, page number, new values, old bytes).
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    __shared__ float lds[4];
    unsigned id = blockIdx.x + a.first;
    const int which = id & 1;
    id >>= 1;
    const int head = id % a.heads;
    id /= a.heads;
    const int t = id % a.touched, b = id / a.touched;
    const Seq s = sequence(a.s, b);
    const int nq = s.nq < s.len ? s.nq : s.len, before = s.len - nq;
    const int blk = (before >> a.s.shift) + t, base = blk << a.s.shift;
    if (nq == 0 || base >= s.len) return;
    const int pid = a.s.table[b * a.s.ld_table + blk];
    if (pid < 0 || pid >= a.s.n_pages) return;
    const int kept = before > base ? before - base : 0;
    const int end = s.len - base < a.s.page ? s.len - base : a.s.page;  // new tokens: [kept, end)
    const int64_t at = int64_t(pid) * a.heads + head;
    // token `slot` of the page is row slot of x (from kept on)
    const int64_t ld = a.tok[which];
    const T *x = static_cast<const T *>(a.src[which]) + (int64_t(s.start) + s.nq - nq + base - before) * ld +
                 head * a.head[which];
    const float old = kept > 0 ? a.scale[which][at] : 0.0f;
    // keys: item i is 16 elements of token i / per; values: 8 elements of 4 tokens, page / 4 items to the elements
    const int per = a.d / 16, quads = a.s.shift - 2;
    const int k_first = kept * per, k_end = end * per, v_items = (a.d / 8) << quads;
    const bool single = end - kept == 1;
    float amax = 0.0f, mine = 0.0f;
    if (single) {  // an element to a thread
        if (int(threadIdx.x) < a.d) mine = float(x[kept * ld + threadIdx.x]);
        amax = __builtin_fabsf(mine);
    } else if (which == 0) {
        for (int i = k_first + threadIdx.x; i < k_end; i += 256) {
            const T *p = x + i / per * ld + i % per * 16;
            float v[2][8];
            load8(p, 8, v[0]);
            load8(p + 8, 8, v[1]);
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = max_nan(__builtin_fabsf(v[e / 8][e % 8]), amax);
        }
    } else {
        for (int i = threadIdx.x; i < v_items; i += 256) {
            const int s0 = (i & ((1 << quads) - 1)) * 4, dd = (i >> quads) * 8;
            if (s0 + 4 <= kept || s0 >= end) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // tokens beside the new ones count the nearest of them again
                const int slot = s0 + e < kept ? kept : s0 + e < end ? s0 + e : end - 1;
                float v[8];
                load8(x + slot * ld + dd, 8, v);
#pragma unroll
                for (int c = 0; c < 8; ++c) amax = max_nan(__builtin_fabsf(v[c]), amax);
            }
        }
    }
    amax = wave_max_nan(amax);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = amax;
    __syncthreads();  // the old scale has been read as well
    amax = max_nan(max_nan(lds[0], lds[1]), max_nan(lds[2], lds[3]));
    const float now = max_nan(old, scale_of(amax).scale);
    const float inv = now > 0.0f ? 1.0f / now : 0.0f, ratio = now > old ? old / now : 1.0f;
    if (threadIdx.x == 0) a.scale[which][at] = now;
    int8_t *page = a.pool[which] + at * a.s.page * a.d;
    const bool grown = kept > 0 && now > old;
    if (single && !grown) {
        const int dd = threadIdx.x;
        if (dd < a.d) page[which ? dd * a.s.page + kept : kept * a.d + dd] = int8_t(quantised(mine, inv));
        return;
    }
    if (which == 0) {
        for (int i = (grown ? 0 : k_first) + threadIdx.x; i < k_end; i += 256) {
            int q[16];
            if (i < k_first) {
                const i32x4 w = *reinterpret_cast<const i32x4 *>(page + i * 16);
#pragma unroll
                for (int e = 0; e < 16; ++e) q[e] = quantised(float(int8_t(uint32_t(w[e / 4]) >> (8 * (e % 4)))), ratio);
            } else {
                const T *p = x + i / per * ld + i % per * 16;
                float v[2][8];
                load8(p, 8, v[0]);
                load8(p + 8, 8, v[1]);
#pragma unroll
                for (int e = 0; e < 16; ++e) q[e] = quantised(v[e / 8][e % 8], inv);
            }
            i32x4 r = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e / 4] |= int(uint32_t(q[e] & 0xFF) << (8 * (e % 4)));
            *reinterpret_cast<i32x4 *>(page + i * 16) = r;
        }
    } else {
        for (int i = threadIdx.x; i < v_items; i += 256) {
            const int s0 = (i & ((1 << quads) - 1)) * 4, dd = (i >> quads) * 8;
            if ((s0 + 4 <= kept && !grown) || s0 >= end) continue;
            uint32_t *p = reinterpret_cast<uint32_t *>(page + dd * a.s.page + s0);
            const int step = a.s.page / 4;
            uint32_t r[8] = {};
            if (s0 < kept || s0 + 4 > end) {  // bytes that are there matter
#pragma unroll
                for (int c = 0; c < 8; ++c) r[c] = p[c * step];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int slot = s0 + e;
                float v[8];
                load8(x + (slot < kept ? kept : slot < end ? slot : end - 1) * ld + dd, 8, v);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    int q = int8_t(r[c] >> (8 * e));
                    if (slot < kept)
                        q = quantised(float(q), ratio);
                    else if (slot < end)
                        q = quantised(v[c], inv);
                    r[c] = (r[c] & ~(0xFFu << (8 * e))) | uint32_t(q & 0xFF) << (8 * e);
                }
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) p[c * step] = r[c];
        }
    }
}

// ------------------------------------------------------------------ attention ------------

constexpr int kMaxSplits = 128;
constexpr int kFewSplits = 12;  // of these a wave joins a row

struct AttnArgs {
    Seqs s;
    const int8_t *k, *v;
    const float *ks, *vs;
    const void *q;
    void *o;
    float *part;  // partial sums of split rows: [token][query head][split][d], then their maxima and sums [..][split][2]
    int64_t q_tok, q_head, o_tok, o_head;
    int q_heads, heads, d, group, causal, window, tiles;
    int64_t units;      // new tokens x query heads
    int splits, chunk;  // a sequence's keys in chunks of `chunk` tokens, `splits` of them at most for any row
    float scale;        // of the scores, with log2(e)
    unsigned first;     // the launch's first workgroup
};

// Four 8-bit integers as FP16, exactly: 0x6400 | u is 1024 + u for a byte u, here the integer + 128.
__device__ __forceinline__ void bytes_to_f16(uint32_t w, f16x2 &lo, f16x2 &hi)
{
    w ^= 0x80808080u;
    const f16x2 bias = {_Float16(1152.0f), _Float16(1152.0f)};
    lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - bias;
    hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - bias;
}

// The same times f, a power of two: one multiply-add in place of the subtraction.
__device__ __forceinline__ f16x8 bytes_to_f16(int w0, int w1, f16x2 f)
{
    const f16x2 bias = f * _Float16(-1152.0f);
    f16x2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = uint32_t(i < 2 ? w0 : w1) ^ 0x80808080u;
        const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w, i & 1 ? 0x04030402u : 0x04010400u);
        v[i] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, u), f, bias);
    }
    return f16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

__device__ __forceinline__ f16x8 bytes_to_f16(int w0, int w1)
{
    f16x2 a, b, c, d;
    bytes_to_f16(uint32_t(w0), a, b);
    bytes_to_f16(uint32_t(w1), c, d);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Keeps the statements of a seldom taken, wave-uniform branch behind it (they are cheap enough for the compiler
// to compute them always and select).
__device__ __forceinline__ void keep_branch() { asm volatile(""); }

// p[0] through the vector memory path.  As a scalar load it would be waited for, memory's latency in full, at every
// barrier that waits for LDS: the two have one counter.
template <typename V>
__device__ __forceinline__ V load_vector(const V *p)
{
    int zero = 0;
    asm volatile("" : "+v"(zero));
    return p[zero];
}

// Asks the compiler for N operand reads, each followed by MFMAS products, in such an order that six reads are under
// way (left to itself it waits for every second one: a read takes as long as three products).
template <int N, int MFMAS>
__device__ __forceinline__ void read_ahead()
{
    constexpr int AHEAD = N < 6 ? N : 6;
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N - AHEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, MFMAS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, AHEAD * MFMAS, 0);
}

// x as the sum of two FP16 values.  x is pinned first: with its last operation folded into the conversion
// (which the compiler does for a multiplication) the higher part would be rounded from another value than the
// lower part is taken from, a whole last place apart at ties.
__device__ __forceinline__ void split_f16(float x, _Float16 &hi, _Float16 &lo)
{
    asm("" : "+v"(x));
    hi = _Float16(x);
    lo = _Float16(x - float(hi));
}

// Rows of one sequence and key head: row = new token * group + query head within the group.  What a tile of
// `count` rows from row0 on sees: keys [begin, end) in all, [all_begin, all_end) by every one of them.
struct Range {
    int begin, end, all_begin, all_end;
};

__device__ __forceinline__ Range row_range(const AttnArgs &a, const Seq &s, int row0, int count)
{
    const int rows = s.nq * a.group;
    const int last = row0 + count - 1 < rows ? row0 + count - 1 : rows - 1;
    const int lo = s.len - s.nq + row0 / a.group, hi = s.len - s.nq + last / a.group;  // their tokens' positions
    Range r;
    r.end = a.causal ? hi + 1 : s.len;
    r.all_end = a.causal ? lo + 1 : s.len;
    r.begin = a.window > 0 && lo >= a.window ? lo - a.window + 1 : 0;
    r.all_begin = a.window > 0 && hi >= a.window ? hi - a.window + 1 : 0;
    return r;
}

// The pages of the tile of 64 tokens from t0 on: one, or with pages of 32 tokens two.  Their numbers are read a
// tile before the rest, which waits for them.  (at: the page and head's place in the cache; a page number
// outside the cache reads as NaN.)
template <bool WHOLE>
struct Pages {
    static constexpr int N = WHOLE ? 1 : 2;
    int number[N];
    int64_t at[N];
    float ks[N], vs[N];

    __device__ __forceinline__ void load_numbers(const AttnArgs &a, int b, int t0)
    {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int blk = (t0 + 32 * h) >> a.s.shift;
            number[h] = blk < a.s.ld_table ? a.s.table[b * a.s.ld_table + blk] : 0;
        }
    }

    __device__ __forceinline__ void load(const AttnArgs &a, int head)
    {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const bool ok = number[h] >= 0 && number[h] < a.s.n_pages;
            at[h] = int64_t(ok ? number[h] : 0) * a.heads + head;
            ks[h] = a.ks[at[h]];
            vs[h] = a.vs[at[h]];
            if (!ok) ks[h] = vs[h] = __builtin_nanf("");
        }
    }
};

// Token of the tile that row i (0..15) of the t-th 16-token tile of the first product stands for.  The
// matrix instruction leaves rows 4 g .. 4 g + 3 to lane group g (lane / 16): so chosen, each group ends up
// with 16 tokens in a row (8 in each half, with pages of 32), which is the operand of the second product.
template <bool WHOLE>
__device__ __forceinline__ int tile_token(int t, int i)
{
    return WHOLE ? i / 4 * 16 + t * 4 + i % 4 : t / 2 * 32 + i / 4 * 8 + t % 2 * 4 + i % 4;
}

// Sixteen rows to a workgroup, whose 4 or 8 waves take tiles of 64 keys in turn and join their sums in LDS at
// the end; one workgroup for each chunk of the keys, whose sums combine_kernel joins where there are
// several.  For few rows: each key and value is read once, by one wave, straight into the registers that
// the matrix instructions take, and the kernel is bound by memory: 64 sequences of up to 8192 tokens, 8 key heads
// of 128: 156 us, 4.5 TB/s (FP32: 163); one of 131001: 62 us, 4.3 TB/s (FP32: 64).  Of 17 to 32 rows each 16 read the
// cache: 16 sequences of 4096 tokens, 8 key heads of 128, 24 rows: 45 us, against 34 for 16 rows.
//
// S^T = K Q^T (tokens down, rows across), P = 2^(S - max), O^T = V^T P^T: S^T's registers are the operand that
// the second product takes, and a row's maximum and sum stay in its lanes.  K and V go in as FP16 integers
// (exact) and the scales are applied to S and to each tile's O.  q is scaled by a power of two to 2^15 and
// P by 2^14, so that FP16 holds q exactly (FP32's: 22 bits, as the sum of two) and P to 11 bits (22)
// down to 2^-28 of the row's largest.  (P in FP16 is what lets one matrix instruction take it; FP32 matrix
// instructions have a sixteenth of the rate.)
template <typename T, int DT, bool WHOLE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 && DT <= 128 ? 3 : 2) void attend_rows_kernel(AttnArgs a)
{
    constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;
    constexpr int PAIRS = DT / 64, DTILES = DT / 16;
    // tiles of values that are loaded beside the keys; the others, for which registers are short, once these are used
    constexpr int EARLY = DT <= 128 ? DTILES : TERMS == 1 ? DTILES / 2 : 0;
    __shared__ float lm[WAVES][16], ll[WAVES][16];
    __shared__ f32x4 lo[WAVES - 1][DTILES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row16 = lane % 16, grp = lane / 16;
    unsigned id = blockIdx.x + a.first;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile = id % a.tiles;
    id /= a.tiles;
    const int head = id % a.heads, b = id / a.heads;
    const Seq s = sequence(a.s, b);
    const int rows = s.nq * a.group;
    if (tile * 16 >= rows) return;
    const Range range = row_range(a, s, tile * 16, 16);
    const int row = tile * 16 + row16;
    const bool live = row < rows;
    const int tq = live ? row / a.group : 0, hq = head * a.group + (live ? row % a.group : 0);
    const int pos = s.len - s.nq + tq;
    const int last = !live ? -1 : a.causal ? pos : s.len - 1, first = a.window > 0 ? pos - a.window + 1 : 0;
    int begin = range.begin & ~63, end = range.end;
    if (a.splits > 1) {
        const int c = range.begin / a.chunk + split;
        if (split > 0 && c * a.chunk >= end) return;
        begin = begin > c * a.chunk ? begin : c * a.chunk;
        end = end < (c + 1) * a.chunk ? end : (c + 1) * a.chunk;
    }

    // q as FP16, scaled by a power of two to magnitudes up to 2^15
    const T *q = static_cast<const T *>(a.q) + (int64_t(s.start) + tq) * a.q_tok + hq * a.q_head;
    float qv[PAIRS][2][8], amax = 0.0f;
#pragma unroll
    for (int p = 0; p < PAIRS; ++p)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = p * 64 + grp * 16 + u * 8;
            load8(q + i, live ? a.d - i : 0, qv[p][u]);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = max_nan(__builtin_fabsf(qv[p][u][e]), amax);
        }
    amax = max_nan(amax, __shfl_xor(amax, 16));
    amax = max_nan(amax, __shfl_xor(amax, 32));
    const int ex = amax > 0.0f && amax < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(amax) : 0;
    const float qs = __builtin_ldexpf(a.scale, -ex);
    f16x8 qf[TERMS][PAIRS][2];
#pragma unroll
    for (int p = 0; p < PAIRS; ++p)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __builtin_ldexpf(qv[p][u][e], ex);
                _Float16 hi, lo;
                split_f16(x, hi, lo);
                qf[0][p][u][e] = hi;
                if constexpr (TERMS == 2) qf[1][p][u][e] = lo;
            }

    const int mask = a.s.page - 1;
    // elements past d are read again from its last 16, so that no read is a branch: q is zero there, and of O they
    // are not stored
    uint32_t k_off[PAIRS];
#pragma unroll
    for (int p = 0; p < PAIRS; ++p) {
        const int i = p * 64 + grp * 16;
        k_off[p] = tile_token<WHOLE>(0, row16) * a.d + (i < a.d ? i : a.d - 16);
    }
    const uint32_t v_off = row16 * a.s.page + grp * (WHOLE ? 16 : 8);
    f32x4 o[DTILES] = {};
    float m = -__builtin_inff(), l = 0.0f;
    Pages<WHOLE> pg;
    int t0 = begin + wave * 64;
    if (t0 < end) pg.load_numbers(a, b, t0);
    for (; t0 < end; t0 += WAVES * 64) {
        pg.load(a, head);
        // lane's keys: of 16 tokens of each 16-token tile, the 16 elements of its group of every 64.  (Addresses are
        // uniform ones and one offset of the lane's: one for each load would be held in registers for the whole loop.)
        const int slot0 = WHOLE ? t0 & mask : 0;
        i32x4 kw[4][PAIRS], vw[DTILES];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int slot = slot0 + (WHOLE ? t * 4 : t % 2 * 4);
            const int8_t *kp = a.k + (pg.at[WHOLE ? 0 : t / 2] * a.s.page + slot) * a.d;
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) kw[t][p] = *reinterpret_cast<const i32x4 *>(kp + k_off[p]);
        }
        // lane's values: row dt * 16 + row16 of V^T, 16 tokens of the group
        auto load_values = [&](int from, int to) {
#pragma unroll
            for (int dt = from; dt < to; ++dt) {
                const int row = dt * 16 < a.d ? dt * 16 : a.d - 16;
                const int8_t *vp = a.v + (pg.at[0] * a.d + row) * a.s.page + slot0;
                if constexpr (WHOLE) {
                    vw[dt] = *reinterpret_cast<const i32x4 *>(vp + v_off);
                } else {
                    const i32x2 w0 = *reinterpret_cast<const i32x2 *>(vp + v_off);
                    const i32x2 w1 =
                        *reinterpret_cast<const i32x2 *>(a.v + (pg.at[1] * a.d + row) * a.s.page + v_off);
                    vw[dt] = i32x4{w0[0], w0[1], w1[0], w1[1]};
                }
            }
        };
        load_values(0, EARLY);
        if (t0 + WAVES * 64 < end) pg.load_numbers(a, b, t0 + WAVES * 64);
        f32x4 sc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            sc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const f16x8 kf = bytes_to_f16(kw[t][p][2 * u], kw[t][p][2 * u + 1]);
#pragma unroll
                    for (int term = 0; term < TERMS; ++term)
                        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[term][p][u], sc[t], 0, 0, 0);
                }
        }
        if constexpr (EARLY < DTILES) {
            __builtin_amdgcn_sched_barrier(0);
            load_values(EARLY, DTILES);
        }
        // lane's scores of row row16: tile t, register r is token tile_token(t, grp * 4 + r)
        const bool masked = t0 < range.all_begin || t0 + 64 > range.all_end;
        float top = m;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float f = pg.ks[WHOLE ? 0 : t / 2] * qs;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[t][r] *= f;
                if (masked) {
                    const int key = t0 + tile_token<WHOLE>(t, grp * 4 + r);
                    sc[t][r] = key <= last && key >= first ? sc[t][r] : -__builtin_inff();
                }
                top = __builtin_fmaxf(top, sc[t][r]);
            }
        }
        top = __builtin_fmaxf(top, __shfl_xor(top, 16));
        top = __builtin_fmaxf(top, __shfl_xor(top, 32));
        // a maximum that rises by less than 1.5 is let be: P stays below 2^15.5, inside FP16
        if (__any(top > m + 1.5f)) {
            keep_branch();
            const float alpha = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < DTILES; ++dt) o[dt] *= alpha;
            m = top;
        }
        const float base = m > -__builtin_inff() ? m - 14.0f : 0.0f;
        f16x8 pf[TERMS][2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f(sc[t][r] - base);
                l += p;
                _Float16 hi, lo;
                split_f16(p, hi, lo);
                pf[0][t / 2][t % 2 * 4 + r] = hi;
                if constexpr (TERMS == 2) pf[1][t / 2][t % 2 * 4 + r] = lo;
            }
        // a page that a row sees nothing of adds nothing to it, whatever its scale; P is 2^14 for m, which O need not
        // have the range for
        float f[Pages<WHOLE>::N];
#pragma unroll
        for (int h = 0; h < Pages<WHOLE>::N; ++h) {
            const int from = t0 + 32 * h, to = from + (WHOLE ? 64 : 32);
            f[h] = last >= from && first < to ? pg.vs[h] * 0x1p-14f : 0.0f;
        }
#pragma unroll
        for (int dt = 0; dt < DTILES; ++dt) {
            f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const f16x8 vf = bytes_to_f16(vw[dt][2 * u], vw[dt][2 * u + 1]);
#pragma unroll
                for (int term = 0; term < TERMS; ++term)
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[term][u], part, 0, 0, 0);
                if (!WHOLE || u == 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[dt][r] = __builtin_fmaf(part[r], f[WHOLE ? 0 : u], o[dt][r]);
                    part = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
            }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    l *= 0x1p-14f;

    // the waves' sums, at the largest maximum of the row
    if (grp == 0) lm[wave][row16] = m;
    __syncthreads();
    float top = lm[0][row16];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = __builtin_fmaxf(top, lm[w][row16]);
    const float f = m > -__builtin_inff() ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
    l *= f;
    if (grp == 0) ll[wave][row16] = l;
    if (wave > 0) {
#pragma unroll
        for (int dt = 0; dt < DTILES; ++dt) lo[wave - 1][dt][lane] = o[dt] * f;
    }
    __syncthreads();
    if (wave > 0 || !live) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) l += ll[w][row16];
    const bool one = a.splits == 1;
    const float inv = one ? (l != 0.0f ? 1.0f / l : 0.0f) : 1.0f;
    const int64_t unit = (int64_t(s.start) + tq) * a.q_heads + hq;
    float *part = a.part + (unit * a.splits + split) * a.d;
    if (!one && grp == 0) {
        float *ml = a.part + a.units * a.splits * a.d + (unit * a.splits + split) * 2;
        ml[0] = top;
        ml[1] = l;
    }
    T *out = static_cast<T *>(a.o) + (int64_t(s.start) + tq) * a.o_tok + hq * a.o_head;
#pragma unroll
    for (int dt = 0; dt < DTILES; ++dt) {
        if (dt * 16 >= a.d) continue;
        f32x4 v = o[dt] * f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += lo[w - 1][dt][lane];
        v *= inv;
        const int i = dt * 16 + grp * 4;
        if (one) {
            const T t[4] = {T(v[0]), T(v[1]), T(v[2]), T(v[3])};
            __builtin_memcpy(out + i, t, sizeof t);
        } else {
            __builtin_memcpy(part + i, &v, 16);
        }
    }
}

// 2^e, or 0 below an FP32 number's range.
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, e > -127 ? uint32_t(e + 127) << 23 : 0u); }

// Places in LDS of the c-th 16 bytes of row r of a K tile (rows of DT FP16) and of a V^T tile (rows of 64).  The
// 16 lanes that read one c of 16 rows get 16 different places modulo the 256 bytes of the banks, and each 8 of
// them 8 different ones modulo 128.
__device__ __forceinline__ int v_place(int r, int c)
{
    return (r >> 1) * 256 + (((r ^ r >> 3) & 1) << 7) + ((c ^ (r & 7)) << 4);
}

template <int DT>
__device__ __forceinline__ int k_place(int r, int c)
{
    return DT == 64 ? v_place(r, c) : r * (DT * 2) + ((c ^ (r & 15)) << 4);
}

// The same for many rows: 32 to a wave, 128 to a team of four waves, which turns each tile of 64 keys into FP16
// once, in LDS (twice the tile: the next one is converted while the waves work on this one).  With two teams each takes
// every other tile, for the same rows, and the first adds the second's sums to its own at the end.  Bound by the
// instructions that a wave issues in turn: of two prompts of 4096 tokens, 32 heads of 128 over 8 key heads, causal,
// BF16 (377 to 392 us, 0.7 PFLOP/s), the matrix units take 29% of the cycles and vector instructions 45%.  Of those, some 370
// for a wave and tile, about 100 turn bytes into FP16 for the next tile, the rest is the softmax: a maximum, a
// multiply-add, an exponential, an addition and half a conversion for each score, and masks and O's rescaling where they are due.
// (The two waves of a SIMD in turns, one multiplying while the other does the rest, and 256 rows to a workgroup were
// slower and the same, against 412 and 378 us at those times.)  One prompt of 2048, 32 heads of 128 over 8, FP32: 122
// us; 16 heads of 256 over 8: BF16 156, FP32 247 us, then 26 for the join.  Heads over 128, and over 64 in FP32, keep
// some values in scratch memory.
//
// 32 x 32 tiles: S^T of 32 tokens and 32 rows leaves a lane 16 scores of one row, the rows of K in LDS in such an
// order that they are two runs of 8 tokens, the operand of O^T = V^T P^T.  The scale of a page's values
// goes into P and the integers, relative to R, set by the largest one so far (uniform; O is held in units of it), until
// scales lie too far apart for that.
template <typename T, int DT, int TEAMS>
__global__ __launch_bounds__(256 * TEAMS, DT > 128 ? 1 : DT <= 64 && TEAMS == 1 && sizeof(T) == 2 ? 3 : 2) void attend_tiles_kernel(AttnArgs a)
{
    constexpr int WAVES = 4, STRIDE = 64 * TEAMS;
    constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;
    constexpr int KSTEPS = DT / 16, DTILES = DT / 32, ROWS = 32 * WAVES;
    constexpr int CHUNKS = 64 * DT / 16, PER = CHUNKS / (64 * WAVES);  // 16-byte pieces of a tile's keys; to a thread
    static_assert(PER >= 1, "a piece for every thread");
    extern __shared__ __align__(16) char smem[];  // for each team two buffers of K [64][DT] and V^T [DT][64]
    const int tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    char *const mem = smem + team * (DT * 512);
    const int col = lane & 31, half = lane >> 5;
    unsigned id = blockIdx.x + a.first;
    const int head = id % a.heads;
    id /= a.heads;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile = a.tiles - 1 - id % a.tiles;  // the tiles with the most keys first
    const int b = id / a.tiles;
    const Seq s = sequence(a.s, b);
    const int rows = s.nq * a.group;
    if (tile * ROWS >= rows) return;
    const Range range = row_range(a, s, tile * ROWS, ROWS);
    const int row0 = tile * ROWS + wave * 32, row = row0 + col;
    const bool live = row < rows;
    const int tq = live ? row / a.group : 0, hq = head * a.group + (live ? row % a.group : 0);
    const int pos = s.len - s.nq + tq;
    const int last = !live ? -1 : a.causal ? pos : s.len - 1, first = a.window > 0 ? pos - a.window + 1 : 0;
    Range mine = {0, 0, 0, 0};
    if (row0 < rows) mine = row_range(a, s, row0, 32);
    int begin = range.begin & ~63, end = range.end;
    if (a.splits > 1) {
        const int c = range.begin / a.chunk + split;
        if (split > 0 && c * a.chunk >= end) return;
        begin = begin > c * a.chunk ? begin : c * a.chunk;
        end = end < (c + 1) * a.chunk ? end : (c + 1) * a.chunk;
    }

    // q as FP16, scaled by a power of two to magnitudes up to 2^15 (and to a positive score scale)
    const T *q = static_cast<const T *>(a.q) + (int64_t(s.start) + tq) * a.q_tok + hq * a.q_head;
    float amax = 0.0f;
    for (int k = 0; k < KSTEPS; ++k) {
        float v[8];
        load8(q + k * 16 + half * 8, live ? a.d - k * 16 - half * 8 : 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(__builtin_fabsf(v[e]), amax);
    }
    amax = max_nan(amax, __shfl_xor(amax, 32));
    const int ex = amax > 0.0f && amax < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(amax) : 0;
    const float qs = __builtin_fabsf(__builtin_ldexpf(a.scale, -ex));
    f16x8 qf[TERMS][KSTEPS];
#pragma unroll
    for (int k = 0; k < KSTEPS; ++k) {
        float v[8];
        load8(q + k * 16 + half * 8, live ? a.d - k * 16 - half * 8 : 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __builtin_ldexpf(a.scale < 0.0f ? -v[e] : v[e], ex);
            _Float16 hi, lo;
            split_f16(x, hi, lo);
            qf[0][k][e] = hi;
            if constexpr (TERMS == 2) qf[1][k][e] = lo;
        }
    }

    // the sequence's row of the page table, and the head's places in the cache (few scalar registers, of which the loop
    // below takes nearly all)
    const int mask = a.s.page - 1, page_bytes = a.s.page * a.d, blocks = int(a.s.ld_table);
    const int *const table = a.s.table + b * a.s.ld_table;
    const int8_t *const keys = a.k + int64_t(head) * page_bytes, *const values = a.v + int64_t(head) * page_bytes;
    const float *const key_scales = a.ks + head, *const value_scales = a.vs + head;
    const uint32_t page_stride = uint32_t(a.heads) * uint32_t(page_bytes);  // below 2^32: 65535 heads of 256 x 256
    i32x4 kw[PER], vw[PER];
    // of the tile from t0 on: the numbers of its halves' pages (read a tile before the rest, which waits for
    // them), where its keys and values begin, and their scales
    int pid[2];
    const int8_t *kp[2], *vp[2];
    float ks[2], vs[2];
    int bad;  // bit h: the page has no place in the cache
    auto load_numbers = [&](int t0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int blk = (t0 + 32 * h) >> a.s.shift;
            pid[h] = load_vector(table + (blk < blocks ? blk : 0));
        }
    };
    auto load_pages = [&](int t0) {
        bad = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = __builtin_amdgcn_readfirstlane(pid[h]);
            const bool ok = n >= 0 && n < a.s.n_pages;
            const uint64_t at = uint64_t(ok ? n : 0) * uint32_t(a.heads), from = uint64_t(ok ? n : 0) * page_stride;
            const int slot = (t0 + 32 * h) & mask;
            kp[h] = keys + from + slot * a.d;
            vp[h] = values + from + slot;
            vs[h] = load_vector(value_scales + at);
            ks[h] = load_vector(key_scales + at);
            bad |= ok ? 0 : 1 << h;
        }
    };
    // a thread's pieces: token tok of the keys, 16 elements from c * 16 on; row dd of the values, 16 tokens from g * 16
    const int kc = tid % (DT / 16), vg = tid % 4;
    int koff[PER], voff[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        // past the head's end the first piece again: those keys meet zeros of q, those values' sums are not stored
        const int dd = (i * 64 * WAVES + tid) / 4;
        koff[i] = (i * 64 * WAVES + tid) / (DT / 16) % 32 * a.d + (kc * 16 < a.d ? kc * 16 : 0);
        voff[i] = (dd < a.d ? dd : 0) * a.s.page + vg % 2 * 16;
    }
    auto load_tile = [&] {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int tok = (i * 64 * WAVES + tid) / (DT / 16);
            kw[i] = *reinterpret_cast<const i32x4 *>((tok < 32 ? kp[0] : kp[1]) + koff[i]);
            vw[i] = *reinterpret_cast<const i32x4 *>((vg < 2 ? vp[0] : vp[1]) + voff[i]);
        }
    };
    // pieces of 16 bytes to two of eight FP16 values; their place in a row is turned by the row's number, so that
    // the reads of sixteen rows at one place spread over the banks
    auto store_tile = [&](char *buf, const uint32_t (&rest)[2]) {
        const f16x2 f = __builtin_bit_cast(f16x2, vg < 2 ? rest[0] : rest[1]);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int tok = (i * 64 * WAVES + tid) / (DT / 16), dd = (i * 64 * WAVES + tid) / 4;
            const int r = (tok & ~12) | (tok & 4) << 1 | (tok & 8) >> 1;  // K's rows: bits 2 and 3 exchanged
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                *reinterpret_cast<f16x8 *>(buf + k_place<DT>(r, kc * 2 + u)) = bytes_to_f16(kw[i][2 * u], kw[i][2 * u + 1]);
                *reinterpret_cast<f16x8 *>(buf + 64 * DT * 2 + v_place(dd, vg * 2 + u)) =
                    bytes_to_f16(vw[i][2 * u], vw[i][2 * u + 1], f);
            }
        }
    };
    // A page's value scale is f 2^e, 0.5 <= f < 1.  P takes f (all its bits stay: rows whose weight lies in many faint
    // keys keep it, and so does the sum of the rounded P), the integers take 2^e relative to R, the power of two above
    // the largest scale so far, exactly: down to 2^-14 a normal FP16 number.  From the first tile with scales
    // further apart on (`spread`) each page's sums are multiplied by its scale in FP32, as for few rows, and R is 2^14,
    // which makes O the numerator itself: a scale however large or small takes nothing from rows that do not
    // see its page.  A page past the keys or before the window, which shares a tile with one that is seen, counts as zeros.
    // (All of it uniform, in scalar registers: R and O's unit as exponents, 126 for 1 and 0 for none yet.)
    constexpr int FAR = 14;
    int big = 0, held = 0;
    float fold[2], ksc[2];
    uint32_t rest[2];  // 2^e / R, twice, as FP16
    int bad_now, spread = 0;
    auto take_scales = [&](int t0) {
        uint32_t vb[2], kb[2];
        bad_now = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            vb[h] = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, vs[h]));
            kb[h] = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, ks[h]));
            const int seen = t0 + 32 * h < range.end && t0 + 32 * h + 32 > range.begin ? 1 : 0;
            const int wrong = bad >> h & 1 || vb[h] >= 0x7F800000u || kb[h] >= 0x7F800000u ? 1 : 0;
            if (wrong || !seen) vb[h] = kb[h] = 0;
            bad_now |= (wrong & seen) << h;
            ksc[h] = __builtin_bit_cast(float, kb[h]);
        }
        const int e0 = vb[0] >> 23, e1 = vb[1] >> 23, most = e0 > e1 ? e0 : e1;
        if (!spread) {
            const bool far = big > 0 && most > big + FAR;
            big = most > big ? most : big;
            spread = far || (e0 > 0 && e0 < big - FAR) || (e1 > 0 && e1 < big - FAR) ? 1 : 0;
            if (spread) big = 126 + FAR;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = int(vb[h] >> 23);  // 0: a scale of zero
            const uint32_t mantissa = vb[h] & 0x7FFFFFu;
            const int at = 126 + e - big;
            if (spread) {
                fold[h] = __builtin_bit_cast(float, e > 0 && at > 0 ? mantissa | uint32_t(at) << 23 : 0u);
                rest[h] = 0x3C003C00u;
            } else {
                fold[h] = __builtin_bit_cast(float, mantissa | 126u << 23);
                rest[h] = e > 0 ? uint32_t(15 + e - big) * 0x04000400u : 0u;
            }
        }
    };

    f32x16 o[DTILES] = {};
    float m = -__builtin_inff(), l = 0.0f;
    int t0 = begin + team * 64, buf = 0;
    if (t0 < end) {
        load_numbers(t0);
        load_pages(t0);
        load_tile();
        load_numbers(t0 + STRIDE);
        take_scales(t0);
        store_tile(mem, rest);
    }
    auto take_turn = [&](auto with_spread) {
        constexpr bool SPREAD = decltype(with_spread)::value;
        const bool more = t0 + STRIDE < end;
        if (more) {
            load_pages(t0 + STRIDE);
            load_tile();
            load_numbers(t0 + 2 * STRIDE);
        }
        __syncthreads();
        const char *kb = mem + buf, *vb = kb + 64 * DT * 2;
        if (t0 < mine.end && t0 + 64 > mine.begin && (TEAMS == 1 || t0 < end)) {
            __builtin_amdgcn_s_setprio(1);
            f32x16 sc[2] = {};
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f16x8 kf = *reinterpret_cast<const f16x8 *>(kb + k_place<DT>(h * 32 + col, k * 2 + half));
#pragma unroll
                    for (int term = 0; term < TERMS; ++term)
                        sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[term][k], sc[h], 0, 0, 0);
                }
            read_ahead<KSTEPS * 2, TERMS>();
            __builtin_amdgcn_s_setprio(0);
            // lane's scores of its row: half h, register r is token t0 + 32 h + r / 8 * 16 + half * 8 + r % 8
            if (t0 < mine.all_begin || t0 + 64 > mine.all_end) {
                keep_branch();
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = t0 + half * 8 + 32 * h + r / 8 * 16 + r % 8;
                        if (!(key <= last && key >= first)) sc[h][r] = -__builtin_inff();
                    }
            }
            if (__builtin_expect(bad_now, 0)) {  // reaches the rows that see the page
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if ((bad_now >> h & 1) && sc[h][r] != -__builtin_inff()) sc[h][r] = __builtin_nanf("");
            }
            float top = m, f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x = -__builtin_inff();
#pragma unroll
                for (int r = 0; r < 16; ++r) x = __builtin_fmaxf(x, sc[h][r]);
                f[h] = __builtin_fmaxf(ksc[h] * qs, 0x1p-120f);  // not 0: it multiplies -Inf
                top = __builtin_fmaxf(top, x * f[h]);
            }
            top = __builtin_fmaxf(top, __shfl_xor(top, 32));
            // a maximum that rises by less than 1.5 is let be: P stays below 2^15.5, inside FP16
            if (__any(top > m + 1.5f) || held != big) {
                keep_branch();
                float alpha = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
                l *= alpha;
                alpha *= power(held > 0 ? held - big : -127);
                held = big;
#pragma unroll
                for (int dt = 0; dt < DTILES; ++dt) o[dt] *= alpha;
                m = top;
            }
            const float base = m > -__builtin_inff() ? m - 14.0f : 0.0f;
            f16x8 pf[TERMS][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // the value scale as part of the exponent, or for FP32 (whose P keeps 22 bits) as a factor
                const float c = SPREAD ? 1.0f : fold[h];
                const float from = TERMS == 1 && !SPREAD ? base - __builtin_amdgcn_logf(c) : base;
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h][r], f[h], -from));
                    if constexpr (TERMS == 2) {
                        sum += p;
                        p *= c;
                    }
                    _Float16 hi, lo;
                    split_f16(p, hi, lo);
                    pf[0][h * 2 + r / 8][r % 8] = hi;
                    if constexpr (TERMS == 2) pf[1][h * 2 + r / 8][r % 8] = lo;
                }
                if constexpr (TERMS == 1) {  // of the rounded P, which the second product takes: two at a time
                    const f16x2 ones = {_Float16(1.0f), _Float16(1.0f)};
#pragma unroll
                    for (int r = 0; r < 16; r += 2)
                        sum = __builtin_amdgcn_fdot2(f16x2{pf[0][h * 2 + r / 8][r % 8], pf[0][h * 2 + r / 8][r % 8 + 1]}, ones,
                                                     sum, false);
                }
                l = __builtin_fmaf(sum, TERMS == 1 && !SPREAD ? __builtin_amdgcn_rcpf(c) : 1.0f, l);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            if constexpr (SPREAD) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int dt = 0; dt < DTILES; ++dt) {
                        f32x16 part = {};
#pragma unroll
                        for (int k = h * 2; k < h * 2 + 2; ++k) {
                            const f16x8 vf = *reinterpret_cast<const f16x8 *>(vb + v_place(dt * 32 + col, k * 2 + half));
#pragma unroll
                            for (int term = 0; term < TERMS; ++term)
                                part = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[term][k], part, 0, 0, 0);
                        }
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[dt][r] = __builtin_fmaf(part[r], fold[h], o[dt][r]);
                        __builtin_amdgcn_sched_barrier(0);  // one `part` at a time
                    }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int dt = 0; dt < DTILES; ++dt) {
                        const f16x8 vf = *reinterpret_cast<const f16x8 *>(vb + v_place(dt * 32 + col, k * 2 + half));
#pragma unroll
                        for (int term = 0; term < TERMS; ++term)
                            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[term][k], o[dt], 0, 0, 0);
                    }
                read_ahead<4 * DTILES, TERMS>();
            }
            __builtin_amdgcn_s_setprio(0);
        }
        if (more) {
            take_scales(t0 + STRIDE);
            store_tile(mem + (buf ^ DT * 256), rest);
        }
        t0 += STRIDE;
        buf ^= DT * 256;
    };
    int turn = begin;  // as many turns for each team
    for (; turn < end && !spread; turn += STRIDE) take_turn(std::false_type());
    for (; turn < end; turn += STRIDE) take_turn(std::true_type());
    // P was 2^14 for m, O in units of `held`: their true values from here on, since another team's (or chunk's) unit may
    // be any other
    l = (l + __shfl_xor(l, 32)) * 0x1p-14f;
    float f = power(held > 0 ? held - 126 - 14 : -127);
    if constexpr (TEAMS == 2) {  // the second team's sums, through LDS, to the first team's
        f32x4 *const so = reinterpret_cast<f32x4 *>(smem);
        float *const sm = reinterpret_cast<float *>(smem + DT * 512);
        __syncthreads();
        if (team == 1) {
#pragma unroll
            for (int dt = 0; dt < DTILES; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    so[(dt * 4 + r) * 256 + tid] =
                        f32x4{o[dt][r * 4], o[dt][r * 4 + 1], o[dt][r * 4 + 2], o[dt][r * 4 + 3]} * f;
            sm[tid] = m;
            sm[256 + tid] = l;
        }
        __syncthreads();
        if (team == 1) return;
        const float m1 = sm[tid], top = __builtin_fmaxf(m, m1);
        const float w0 = m > -__builtin_inff() ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
        const float w1 = m1 > -__builtin_inff() ? __builtin_amdgcn_exp2f(m1 - top) : 0.0f;
        l = l * w0 + sm[256 + tid] * w1;
        const float f0 = f * w0;
#pragma unroll
        for (int dt = 0; dt < DTILES; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = __builtin_fmaf(o[dt][r], f0, so[(dt * 4 + r / 4) * 256 + tid][r % 4] * w1);
        m = top;
        f = 1.0f;
    }
    if (!live) return;
    const bool one = a.splits == 1;
    if (one) f *= l != 0.0f ? 1.0f / l : 0.0f;
    const int64_t unit = (int64_t(s.start) + tq) * a.q_heads + hq;
    float *part = a.part + (unit * a.splits + split) * a.d;
    if (!one && half == 0) {
        float *ml = a.part + a.units * a.splits * a.d + (unit * a.splits + split) * 2;
        ml[0] = m;
        ml[1] = l;
    }
    T *out = static_cast<T *>(a.o) + (int64_t(s.start) + tq) * a.o_tok + hq * a.o_head;
#pragma unroll
    for (int dt = 0; dt < DTILES; ++dt)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const int i = dt * 32 + r4 * 8 + half * 4;
            if (i >= a.d) continue;
            const f32x4 v = f32x4{o[dt][r4 * 4], o[dt][r4 * 4 + 1], o[dt][r4 * 4 + 2], o[dt][r4 * 4 + 3]} * f;
            if (one) {
                const T t[4] = {T(v[0]), T(v[1]), T(v[2]), T(v[3])};
                __builtin_memcpy(out + i, t, sizeof t);
            } else {
                *reinterpret_cast<f32x4 *>(part + i) = v;
            }
        }
}

// Joins the chunks' sums of rows that have few chunks: a wave to a row, one element of O or more to a lane (2048 rows
// of 4 chunks of 128: 5.8 us).
template <typename T>
__global__ __launch_bounds__(256) void combine_few_kernel(AttnArgs a, int span, int64_t count)
{
    int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int hq = int(id % a.q_heads);
    id /= a.q_heads;
    const int tq = int(id % a.s.max_new), b = int(id / a.s.max_new);
    const Seq s = sequence(a.s, b);
    if (tq >= s.nq) return;
    const int lane = threadIdx.x & 63;
    const int row = tq * a.group + hq % a.group;
    const Range tile = row_range(a, s, row / span * span, span), own = row_range(a, s, row, 1);
    const int c0 = tile.begin / a.chunk;
    const int lo = own.begin / a.chunk - c0, hi = own.end > own.begin ? (own.end - 1) / a.chunk - c0 + 1 : lo;
    const int64_t unit = (int64_t(s.start) + tq) * a.q_heads + hq;
    const float *part = a.part + unit * a.splits * a.d;
    const float *ml = a.part + a.units * a.splits * a.d + unit * a.splits * 2;
    float m = -__builtin_inff(), l = 0.0f;
    if (lo + lane < hi) {  // hi - lo <= 64
        m = ml[(lo + lane) * 2];
        l = ml[(lo + lane) * 2 + 1];
    }
    const float top = wave_max_nan(m);
    const float w = m > -__builtin_inff() ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
    l = wave_sum(l * w);
    float acc[4] = {};
    for (int c = lo; c < hi; c += 4) {  // four chunks' loads under way; past the last one w is 0
        float v[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[u][e] = c + u < hi && e * 64 + lane < a.d ? part[int64_t(c + u) * a.d + e * 64 + lane] : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float wc = __shfl(w, c - lo + u);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(v[u][e], wc, acc[e]);
        }
    }
    T *out = static_cast<T *>(a.o) + (int64_t(s.start) + tq) * a.o_tok + hq * a.o_head;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < a.d) out[e * 64 + lane] = T(l != 0.0f ? acc[e] / l : 0.0f);
}

// Joins the chunks' sums of a row (one workgroup): O = sum w_c O_c / sum w_c l_c, w_c = 2^(m_c - max).  The
// weights go to LDS, then four elements of each chunk's O to a thread, the threads of a row of O in
// groups that take the chunks in turn (32 rows of 128 chunks: 6.3 us).  `span`: rows of a tile of the kernel that wrote them.
template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(AttnArgs a, int span)
{
    __shared__ float lds[4], weight[kMaxSplits + 1];
    __shared__ f32x4 lacc[256];
    unsigned id = blockIdx.x;
    const int hq = id % a.q_heads;
    id /= a.q_heads;
    const int tq = id % a.s.max_new, b = id / a.s.max_new;
    const Seq s = sequence(a.s, b);
    if (tq >= s.nq) return;
    const int tid = threadIdx.x;
    const int row = tq * a.group + hq % a.group;
    const Range tile = row_range(a, s, row / span * span, span), own = row_range(a, s, row, 1);
    // chunks that hold a key of the row, from the tile's first one on
    const int c0 = tile.begin / a.chunk;
    const int lo = own.begin / a.chunk - c0, hi = own.end > own.begin ? (own.end - 1) / a.chunk - c0 + 1 : lo;
    const int64_t unit = (int64_t(s.start) + tq) * a.q_heads + hq;
    const float *part = a.part + unit * a.splits * a.d;
    const float *ml = a.part + a.units * a.splits * a.d + unit * a.splits * 2;
    float m = -__builtin_inff(), l = 0.0f;
    if (lo + tid < hi) {  // hi - lo <= kMaxSplits + 1 <= 256
        m = ml[(lo + tid) * 2];
        l = ml[(lo + tid) * 2 + 1];
    }
    float top = wave_max_nan(m);
    if ((tid & 63) == 0) lds[tid >> 6] = top;
    __syncthreads();
    top = max_nan(max_nan(lds[0], lds[1]), max_nan(lds[2], lds[3]));
    const float w = m > -__builtin_inff() ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
    if (lo + tid < hi) weight[tid] = w;
    l = wave_sum(l * w);
    __syncthreads();
    if ((tid & 63) == 0) lds[tid >> 6] = l;
    const int quads = a.d / 4, groups = 256 / quads, quad = tid % quads, g = tid / quads;
    f32x4 acc = {};
    if (g < groups) {
#pragma unroll 4
        for (int c = lo + g; c < hi; c += groups)
            acc += *reinterpret_cast<const f32x4 *>(part + int64_t(c) * a.d + quad * 4) * weight[c - lo];
    }
    lacc[tid] = acc;
    __syncthreads();
    if (tid >= quads) return;
    l = lds[0] + lds[1] + lds[2] + lds[3];
    for (int i = 1; i < groups; ++i) acc += lacc[i * quads + tid];
    T *out = static_cast<T *>(a.o) + (int64_t(s.start) + tq) * a.o_tok + hq * a.o_head + tid * 4;
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    const T t[4] = {T(acc[0] * inv), T(acc[1] * inv), T(acc[2] * inv), T(acc[3] * inv)};
    __builtin_memcpy(out, t, sizeof t);
}

// How the attention of a call is laid out over workgroups: by sixteen rows, or for more than 32 rows of a
// sequence and key head by `span`.
struct AttnPlan {
    int span, tiles, splits, chunk;
    bool wide;  // workgroups of 8 waves, not 4: all on 16 rows, or two teams on 128
    size_t bytes;
};

AttnPlan plan_attention(const amsim_cache8 *c, int64_t batch, int64_t q_heads, int64_t total_new, int64_t max_new,
                        int64_t max_len, int64_t window)
{
    const int64_t group = q_heads / c->heads, rows = max_new * group;
    AttnPlan p{};
    p.span = rows <= 32 ? 16 : 128;
    p.tiles = int(ceil_div(rows, p.span));
    // keys that a tile's rows see, and workgroups without splitting them
    const int64_t seen = window > 0 && window + p.span < max_len ? window + p.span : max_len;
    const int64_t units = batch * c->heads * p.tiles;
    // splits so that some 2048 workgroups run, with 256 keys at least for each; of those with many rows (whose sums
    // are more to join: 49 against 57 us for a chunk of 509 tokens over 1024 keys each, by one team) one for each compute
    // unit, with 1024 keys, or for large heads (one team) two
    const int64_t least = p.span == 16 ? 256 : 1024;
    int64_t splits = units > 0 ? (p.span == 16 ? 2048 : c->head_dim <= 128 ? 256 : 512) / units : 1;
    const int64_t each = p.span == 16 ? ceil_div(seen, least) : seen / least;
    const int64_t most = each < kMaxSplits ? each : kMaxSplits;
    splits = splits > most ? most : splits;
    // few rows whose keys and values are read by one workgroup about as fast as by several, whose sums then have to
    // be joined by another kernel: 256 KB of them, by twice the waves (1000 keys of 128: 14.3 against 15.5 us for 8
    // workgroups, 18.9 against 25.0 for 256, 31.8 against 36.4 for 512; more of them fill the GPU with 4 waves each)
    p.wide = p.span == 16 && seen > 256 && seen * c->head_dim <= 1 << 17 && units <= 512;
    if (splits < 1 || p.wide) splits = 1;
    // two teams of waves share a tile of rows' keys where that leaves no compute unit without a workgroup (times with
    // the append): a chunk of 509 tokens, window 1024, 12 heads of 64, 3 sequences: 40 against 49 us; 2048 tokens of
    // 12 heads of 64: 50 against 62 us for two chunks of keys without
    if (p.span > 16) p.wide = c->head_dim <= 128 && seen > 64 && units * splits <= 256;
    p.chunk = int(ceil_div(ceil_div(seen, splits), 256) * 256);
    if (p.chunk < 256) p.chunk = 256;
    // a window begins anywhere inside a chunk
    p.splits = splits == 1 ? 1 : int(ceil_div(seen, p.chunk)) + (seen < max_len ? 1 : 0);
    p.bytes = p.splits > 1 ? size_t(total_new) * size_t(q_heads) * size_t(p.splits) * size_t(c->head_dim + 2) * 4 : 0;
    return p;
}

template <typename T, int DT, int TEAMS>
int launch_tiles_of(const AttnArgs &a, unsigned groups, hipStream_t st)
{
    constexpr int kLds = TEAMS * DT * 512;
    // more than 64 KB of LDS has to be asked for, once
    static const hipError_t asked = hipFuncSetAttribute(reinterpret_cast<const void *>(attend_tiles_kernel<T, DT, TEAMS>),
                                                        hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (asked != hipSuccess) return AMSIM_ERR_HIP;
    hipLaunchKernelGGL((attend_tiles_kernel<T, DT, TEAMS>), dim3(groups), dim3(256 * TEAMS), kLds, st, a);
    return AMSIM_OK;
}

template <typename T>
int launch_tiles(const AttnArgs &a, bool wide, unsigned groups, hipStream_t st)
{
    if (a.d <= 64) return wide ? launch_tiles_of<T, 64, 2>(a, groups, st) : launch_tiles_of<T, 64, 1>(a, groups, st);
    if (a.d <= 128) return wide ? launch_tiles_of<T, 128, 2>(a, groups, st) : launch_tiles_of<T, 128, 1>(a, groups, st);
    return launch_tiles_of<T, 256, 1>(a, groups, st);
}

template <typename T>
void launch_rows(const AttnArgs &a, bool wide, unsigned groups, hipStream_t st)
{
#define ROWS(DT) \
    do { \
        if (a.s.page >= 64 && wide) \
            hipLaunchKernelGGL((attend_rows_kernel<T, DT, true, 8>), dim3(groups), dim3(512), 0, st, a); \
        else if (a.s.page >= 64) \
            hipLaunchKernelGGL((attend_rows_kernel<T, DT, true, 4>), dim3(groups), dim3(256), 0, st, a); \
        else if (wide) \
            hipLaunchKernelGGL((attend_rows_kernel<T, DT, false, 8>), dim3(groups), dim3(512), 0, st, a); \
        else \
            hipLaunchKernelGGL((attend_rows_kernel<T, DT, false, 4>), dim3(groups), dim3(256), 0, st, a); \
    } while (0)
    if (a.d <= 64)
        ROWS(64);
    else if (a.d <= 128)
        ROWS(128);
    else
        ROWS(256);
#undef ROWS
}

// ------------------------------------------------------------------ checks ---------------

int check_cache(const amsim_cache8 *c)
{
    if (!c || c->pages < 0 || c->heads < 1) return AMSIM_ERR_INVALID_ARG;
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256)
        return AMSIM_ERR_UNSUPPORTED;
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16) return AMSIM_ERR_UNSUPPORTED;
    if (c->pages >= int64_t(1) << 31 || c->heads > 65535) return AMSIM_ERR_UNSUPPORTED;
    if (c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return AMSIM_ERR_INVALID_ARG;
    if ((uintptr_t(c->k) | uintptr_t(c->v)) & 15) return AMSIM_ERR_INVALID_ARG;
    return AMSIM_OK;
}

int check_seqs(const amsim_cache8 *c, int64_t batch, const int *table, int64_t ld_table, const int *lengths,
               const int *starts, int64_t total_new, int64_t max_new, int64_t max_len, Seqs &s)
{
    if (batch < 0 || ld_table < 0 || total_new < 0 || max_new < 0 || max_len < 0) return AMSIM_ERR_INVALID_ARG;
    const int64_t lim = int64_t(1) << 30;
    if (batch >= lim || total_new >= lim || max_len >= lim || ld_table >= lim) return AMSIM_ERR_UNSUPPORTED;
    if (batch > 0 && (!lengths || !starts || (ld_table > 0 && !table))) return AMSIM_ERR_INVALID_ARG;
    int shift = 5;
    while ((1 << shift) < c->page_tokens) ++shift;
    s = Seqs{table, lengths, starts, ld_table, int(batch), int(max_new < total_new ? max_new : total_new),
             int(total_new), int(c->pages), c->page_tokens, shift, max_len};
    return AMSIM_OK;
}

}  // namespace

extern "C" {

int amsim_cache_append(const amsim_cache8 *cache, int64_t batch, const int32_t *page_table, int64_t ld_table,
                       const int32_t *lengths, const int32_t *starts, int64_t total_new, int64_t max_new, int dtype,
                       const void *k, int64_t k_token, int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
                       void *stream)
{
    int rc = check_cache(cache);
    if (rc != AMSIM_OK) return rc;
    if (!valid_type(dtype)) return AMSIM_ERR_INVALID_ARG;
    AppendArgs a{};
    const int64_t most = (int64_t(1) << 30) - 1;
    rc = check_seqs(cache, batch, page_table, ld_table, lengths, starts, total_new, max_new, most, a.s);
    if (rc != AMSIM_OK) return rc;
    if (batch == 0 || total_new == 0 || max_new == 0 || ld_table == 0 || cache->pages == 0) return AMSIM_OK;
    if (!k || !v) return AMSIM_ERR_INVALID_ARG;
    a.src[0] = k, a.src[1] = v;
    a.tok[0] = k_token, a.tok[1] = v_token;
    a.head[0] = k_head, a.head[1] = v_head;
    a.pool[0] = cache->k, a.pool[1] = cache->v;
    a.scale[0] = cache->k_scale, a.scale[1] = cache->v_scale;
    a.heads = cache->heads, a.d = cache->head_dim;
    // new tokens that start inside a page reach into one page more
    a.touched = int(ceil_div(a.s.max_new - 1, a.s.page) + 1);
    const int64_t lim = int64_t(1) << 31;
    if (2 * batch * a.heads >= lim || 2 * batch * a.heads * a.touched >= lim) return AMSIM_ERR_UNSUPPORTED;
    const int64_t groups = 2 * batch * a.heads * a.touched;
    return with_type(dtype, [&](auto t) {
        in_launches(groups, [&](int64_t first, unsigned count) {
            a.first = unsigned(first);
            hipLaunchKernelGGL((append_kernel<decltype(t)>), dim3(count), dim3(256), 0, static_cast<hipStream_t>(stream), a);
        });
        return launch_status();
    });
}

int amsim_cache_attention_workspace_size(const amsim_cache8 *cache, int64_t batch, int64_t q_heads, int64_t total_new,
                                         int64_t max_new, int64_t max_len, int64_t window, size_t *bytes)
{
    const int rc = check_cache(cache);
    if (rc != AMSIM_OK) return rc;
    if (!bytes || batch < 0 || q_heads < 1 || total_new < 0 || max_new < 0 || max_len < 0 || window < 0)
        return AMSIM_ERR_INVALID_ARG;
    if (q_heads % cache->heads) return AMSIM_ERR_INVALID_ARG;
    const int64_t lim = int64_t(1) << 30;
    if (batch >= lim || q_heads / cache->heads > 65535 || total_new >= lim || max_len >= lim ||
        (max_new < total_new ? max_new : total_new) * (q_heads / cache->heads) >= lim)
        return AMSIM_ERR_UNSUPPORTED;
    // what the plan multiplies stays within 64 bits
    const int64_t tiles = ceil_div((max_new < total_new ? max_new : total_new) * (q_heads / cache->heads), 16);
    if (batch * cache->heads >= lim || batch * cache->heads * tiles >= lim || total_new * q_heads >= lim << 10)
        return AMSIM_ERR_UNSUPPORTED;
    *bytes = plan_attention(cache, batch, q_heads, total_new, max_new < total_new ? max_new : total_new, max_len, window)
                 .bytes;
    return AMSIM_OK;
}

int amsim_cache_attention(const amsim_cache8 *cache, int64_t batch, const int32_t *page_table, int64_t ld_table,
                          const int32_t *lengths, const int32_t *starts, int64_t total_new, int64_t max_new,
                          int64_t max_len, int dtype, int64_t q_heads, const void *q, int64_t q_token, int64_t q_head,
                          float scale, int causal, int64_t window, void *out, int64_t out_token, int64_t out_head,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    int rc = amsim_cache_attention_workspace_size(cache, batch, q_heads, total_new, max_new, max_len, window, &need);
    if (rc != AMSIM_OK) return rc;
    if (!valid_type(dtype) || (window > 0 && !causal)) return AMSIM_ERR_INVALID_ARG;
    scale *= 1.44269504f;
    if (!(__builtin_fabsf(scale) < __builtin_inff())) return AMSIM_ERR_INVALID_ARG;
    AttnArgs a{};
    rc = check_seqs(cache, batch, page_table, ld_table, lengths, starts, total_new, max_new, max_len, a.s);
    if (rc != AMSIM_OK) return rc;
    if (batch == 0 || total_new == 0 || max_new == 0) return AMSIM_OK;
    if (!q || !out || cache->pages == 0) return AMSIM_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need)) return AMSIM_ERR_WORKSPACE;
    if (uintptr_t(workspace) & 15) return AMSIM_ERR_INVALID_ARG;
    const AttnPlan p = plan_attention(cache, batch, q_heads, total_new, a.s.max_new, max_len, window);
    a.k = cache->k, a.v = cache->v, a.ks = cache->k_scale, a.vs = cache->v_scale;
    a.q = q, a.o = out, a.part = static_cast<float *>(workspace);
    a.q_tok = q_token, a.q_head = q_head, a.o_tok = out_token, a.o_head = out_head;
    a.q_heads = int(q_heads), a.heads = cache->heads, a.d = cache->head_dim, a.group = int(q_heads / cache->heads);
    a.causal = causal != 0, a.window = int(window < (int64_t(1) << 30) ? window : 0);
    a.scale = scale;
    a.units = total_new * q_heads;
    a.tiles = p.tiles, a.splits = p.splits, a.chunk = p.chunk;
    const int64_t lim = int64_t(1) << 31, groups = batch * a.heads * a.tiles * a.splits;
    const int64_t joins = p.splits > 1 ? batch * a.s.max_new * a.q_heads : 0;
    if (groups >= lim || joins >= lim) return AMSIM_ERR_UNSUPPORTED;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const hipStream_t st = static_cast<hipStream_t>(stream);
        int done = AMSIM_OK;
        in_launches(groups, [&](int64_t first, unsigned count) {
            a.first = unsigned(first);
            if (p.span == 16)
                launch_rows<T>(a, p.wide, count, st);
            else if (done == AMSIM_OK)
                done = launch_tiles<T>(a, p.wide, count, st);
        });
        if (done != AMSIM_OK) return done;
        if (joins > 0 && p.splits <= kFewSplits)
            hipLaunchKernelGGL((combine_few_kernel<T>), dim3(static_cast<unsigned>(ceil_div(joins, 4))), dim3(256), 0, st,
                               a, p.span, joins);
        else if (joins > 0)
            hipLaunchKernelGGL((combine_kernel<T>), dim3(static_cast<unsigned>(joins)), dim3(256), 0, st, a, p.span);
        return launch_status();
    });
}

}  // extern "C"
