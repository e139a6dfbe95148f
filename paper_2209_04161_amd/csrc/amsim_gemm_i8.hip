// amsim_gemm_i8.hip -- product of 8-bit integer matrices with a scale for each token and channel:
//   C[i][j] = (sum_k a[i][k] b[j][k]) a_scale[i] b_scale[j] + bias[j],
// the sum in 32-bit integers on the matrix cores (exact: k < 2^17), the scaling in FP32, rounded once
// to C's type.
#include <type_traits>

#include "amsim_q8.h"

namespace {

using namespace amsim_q8;

constexpr int64_t kMaxK = (int64_t(1) << 17) - 1;  // 128 * 128 * k stays below 2^31
constexpr int kStep = 128;                           // bytes of k that a tile takes at a time

struct GemmArgs {
    const int8_t *a, *b;
    const float *as, *bs, *bias;
    void *c;
    int *part;  // [split][m][n] integer sums of split products
    int64_t lda, ldb, ldc;
    int m, n, k;
    int tiles_m, tiles_n, splits, per;  // per: steps of k to a split
};

// Sixteen bytes from p on, whatever its alignment, as the whole words that hold them.  (For lanes that each read a
// row of their own, 16-byte loads at addresses that are not multiples of 4 are slower: 62 against 31 us for
// 16 x 8192 x 8191.)
struct Words {
    i32x4 w;
    int next;

    __device__ __forceinline__ void load(const int8_t *p)
    {
        const int shift = int(uintptr_t(p) & 3);
        const int *q = reinterpret_cast<const int *>(p - shift);
        __builtin_memcpy(&w, q, 16);
        next = q[shift ? 4 : 3];  // the word after, if it holds any of them
    }

    __device__ __forceinline__ i32x4 bytes(int shift) const  // shift: the address modulo 4
    {
        i32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = int(__builtin_amdgcn_alignbyte(uint32_t(e < 3 ? w[e + 1] : next), uint32_t(w[e]), shift));
        return v;
    }
};

// Up to sixteen bytes of a row from p on, `left` of them inside it; the others are zeros.
__device__ __forceinline__ i32x4 load_part(const int8_t *p, int left)
{
    uint64_t w[2] = {0, 0};
#pragma unroll 1
    for (int e = 0; e < 16 && e < left; ++e) {
        const uint64_t x = uint64_t(uint8_t(p[e])) << (8 * (e & 7));
        w[0] |= e < 8 ? x : 0;
        w[1] |= e < 8 ? 0 : x;
    }
    return i32x4{int(w[0]), int(w[0] >> 32), int(w[1]), int(w[1] >> 32)};
}

// All sixteen where they are inside.  Where 8 lanes read 128 bytes in a row, addresses of any alignment are served
// faster than the words around them put together (17 against 23 us for 64 x 8192 x 4099).
__device__ __forceinline__ i32x4 load16(const int8_t *p, int left)
{
    if (left < 16) return load_part(p, left);
    i32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// N results of row i from column j on, from their integer sums.
template <typename T, int N>
__device__ __forceinline__ void store_row(const GemmArgs &g, int i, int j, const int (&sum)[N])
{
    if (i >= g.m || j >= g.n) return;
    const float as = g.as[i];
    T *c = static_cast<T *>(g.c) + i * g.ldc + j;
    T t[N];
    if (j + N <= g.n) {
        float bs[N], bias[N] = {};
        __builtin_memcpy(bs, g.bs + j, sizeof bs);
        if (g.bias) __builtin_memcpy(bias, g.bias + j, sizeof bias);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float v = float(sum[e]) * as * bs[e];
            if (g.bias) v += bias[e];
            t[e] = T(v);
        }
        __builtin_memcpy(c, t, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (j + e < g.n) {
                float v = float(sum[e]) * as * g.bs[j + e];
                if (g.bias) v += g.bias[j + e];
                c[e] = T(v);
            }
    }
}

// Copies 16 bytes a lane from global memory to LDS at base + lane * 16, without passing through registers.
__device__ __forceinline__ void copy_to_lds(const int8_t *p, int8_t *base)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p,
                                     (__attribute__((address_space(3))) void *)base, 16, 0, 0);
}

// Waits until at most N of the wave's copies are under way and its reads of LDS are done, and then for the other
// waves.  (A __syncthreads would wait for all of the copies.)
template <int N>
__device__ __forceinline__ void wait_copies()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A BM x BN tile of C (tokens x channels) to a workgroup of WM x WN waves.  k is taken in steps of 128 bytes (whole
// cache lines: with steps of 64 the tile's reads were twice as many requests to the L2), each in two halves.
// ALIGNED (rows at multiples of 16 bytes): through a ring of STAGES buffers in LDS; the operands of a half are read
// into registers while the half before is multiplied, and the copies of the next STAGES - 1 steps are under
// way.  Otherwise (and the last step, where it is not whole) through registers and two buffers.
// Tiles of 256: 8192 x 8192 x 8192 465 to 502 us, 2.2 to 2.4 POP/s, 8192 x 8192 x 4096 264 to 284 us, 1.9 to 2.1 POP/s,
// as the library's product (the matrix units are busy 49% of the cycles); of 128: 2048 x 2048 x 4096 29 us, 1.2
// POP/s, one workgroup of four waves to a compute unit; of 64: 48 x 16384 x 4096 19.5 us, 3.4 TB/s of weights, bound by memory
// (13 us where the weights are in the last-level cache), 1000 x 777 x 1111 13 us, bound by latency.
//
// In LDS a row has 128 bytes, 8 pieces of 16, whose order is turned by the row's number: a 16-byte read of a wave is
// served 16 lanes at a time, lanes 0-3, 12-15, 20-23 and 24-27 first, then 4-11, 16-19 and 28-31, and these lie in
// 16 different places modulo the 256 bytes of the banks.  The channels are the instruction's rows: lane group g
// (lane / 16) gets rows 4 g .. 4 g + 3 of each of a wave's TN 16-row tiles, which stand for channels 4 TN g
// + 4 s + .. of the wave's, so that a lane ends up with 4 TN channels in a row of one token.
template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN, 2) void gemm_tile_kernel(GemmArgs g)
{
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16, ROWS = BM + BN, STAGE = ROWS * kStep;
    constexpr int WAVES = WM * WN, COPIES = ROWS / 8 / WAVES;  // pieces of a step for each lane
    constexpr int COPIES_A = BM / 8 / WAVES;
    constexpr int SH = TN == 8 ? 5 : TN == 4 ? 4 : 3;
    static_assert(TN == 8 || TN == 4 || TN == 2, "the order of the pieces is made for these");
    static_assert((STAGES & (STAGES - 1)) == 0 && STAGES >= 2, "a ring of a power of two");
    extern __shared__ __align__(16) int8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // consecutive workgroups go to the 8 XCDs in turn: each XCD takes a run of tiles, in columns of 8 tiles of
    // tokens, so that what its workgroups read at a time stays in its L2
    const int tiles = g.tiles_m * g.tiles_n;
    int id = blockIdx.x % tiles;
    const int split = blockIdx.x / tiles;
    const int whole = tiles / 8 * 8;
    if (id < whole) id = id % 8 * (whole / 8) + id / 8;
    const int group = id / (8 * g.tiles_n), in = id % (8 * g.tiles_n);
    const int high = g.tiles_m - group * 8 < 8 ? g.tiles_m - group * 8 : 8;
    const int i0 = (group * 8 + in % high) * BM, j0 = in / high * BN;

    const int steps = (g.k + kStep - 1) / kStep;
    const int t0 = split * g.per, t1 = t0 + g.per < steps ? t0 + g.per : steps;

    // the lane's pieces of a step, from the tile's first rows on; rows past the matrix repeat its last one
    const int8_t *const base[2] = {g.a + i0 * g.lda, g.b + j0 * g.ldb};
    typename std::conditional<ALIGNED, uint32_t, int64_t>::type off[COPIES];
    int piece[COPIES];
#pragma unroll
    for (int q = 0; q < COPIES; ++q) {
        int r = (q * WAVES + wave) * 8 + lane / 8;
        if (q < COPIES_A) {
            piece[q] = ((lane & 7) ^ (r >> 1 & 7)) * 16;
            r = r < g.m - i0 ? r : g.m - i0 - 1;
            off[q] = r * g.lda + piece[q];
        } else {
            r -= BM;
            piece[q] = ((lane & 7) ^ ((r >> 1 & 1) | (r >> SH & 3) << 1)) * 16;
            r = r < g.n - j0 ? r : g.n - j0 - 1;
            off[q] = r * g.ldb + piece[q];
        }
    }
    auto load = [&](int t, i32x4 (&v)[COPIES]) {
        if (t * kStep + kStep <= g.k) {
#pragma unroll
            for (int q = 0; q < COPIES; ++q)
                __builtin_memcpy(&v[q], base[q >= COPIES_A] + int64_t(t) * kStep + off[q], 16);
        } else {
#pragma unroll
            for (int q = 0; q < COPIES; ++q)
                v[q] = load16(base[q >= COPIES_A] + int64_t(t) * kStep + off[q], g.k - t * kStep - piece[q]);
        }
    };
    auto store = [&](int t, const i32x4 (&v)[COPIES]) {
#pragma unroll
        for (int q = 0; q < COPIES; ++q)
            *reinterpret_cast<i32x4 *>(smem + (t & 1) * STAGE + (q * WAVES + wave) * 1024 + lane * 16) = v[q];
    };

    // where the wave's operands lie in a step: the lane's row of each tile, and its piece of each half
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const int ra = (wm + lane % 16) * kStep, rb = (BM + wn + lane % 16 / 4 * (4 * TN) + lane % 4) * kStep;
    const int at[2] = {(lane / 16 ^ lane % 16 >> 1) * 16, (lane / 16 + 4 ^ lane % 16 >> 1) * 16};
    i32x4 acc[TN][TM] = {};
    i32x4 fa[2][TM], fb[2][TN];
    auto read = [&](int t, int half) {
        const int8_t *from = smem + (t & (STAGES - 1)) * STAGE + at[half];
#pragma unroll
        for (int i = 0; i < TN; ++i) fb[half][i] = *reinterpret_cast<const i32x4 *>(from + rb + i * (4 * kStep));
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[half][i] = *reinterpret_cast<const i32x4 *>(from + ra + i * (16 * kStep));
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
            for (int s = 0; s < TN; ++s)
                acc[s][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[half][s], fa[half][t], acc[s][t], 0, 0, 0);
    };
    int tail = t0;
    if constexpr (ALIGNED) {
        const int end = t1 < g.k / kStep ? t1 : g.k / kStep;  // steps that are whole
        tail = end;
        const int n = end - t0;
        auto copy = [&](int t) {
            const int64_t from = int64_t(t0 + t) * kStep;
            int8_t *to = smem + (t & (STAGES - 1)) * STAGE + wave * 1024;
#pragma unroll
            for (int q = 0; q < COPIES; ++q) copy_to_lds(base[q >= COPIES_A] + from + off[q], to + q * (WAVES * 1024));
        };
        if constexpr (WAVES == 8) {
            // Two waves to a SIMD, which take turns: while one multiplies the other reads its operands of the next half,
            // with a barrier between the phases.  Waves 4-7 are one phase behind.
            const bool behind = wave >= 4;
            auto phase = [](bool lds, bool copies) {
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" ::: "memory");
                if (lds) __builtin_amdgcn_s_waitcnt(0xC07F);
                if (copies) __builtin_amdgcn_s_waitcnt(0x0F70);
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            };
            if (n > 0) {
                copy(0);
                phase(false, true);
                if (n > 1) copy(1);
                if (behind) phase(false, false);
                for (int t = 0; t < n; ++t) {
                    read(t, 0);
                    if (t > 0 && t + 1 < n) copy(t + 1);  // over step t - 1, which all have read
                    phase(true, false);
                    __builtin_amdgcn_s_setprio(1);
                    multiply(0);
                    __builtin_amdgcn_s_setprio(0);
                    phase(false, false);
                    read(t, 1);
                    phase(true, behind);  // step t + 1 is there for the others once these waves' part is
                    __builtin_amdgcn_s_setprio(1);
                    multiply(1);
                    __builtin_amdgcn_s_setprio(0);
                    phase(false, !behind);
                }
                if (!behind) phase(false, false);
            }
        } else if (n > 0) {
            for (int t = 0; t < STAGES && t < n; ++t) copy(t);
            if (n >= STAGES)
                wait_copies<COPIES *(STAGES - 1)>();
            else
                wait_copies<0>();
            read(0, 0);
            int t = 0;
            for (; t + STAGES < n; ++t) {
                read(t, 1);
                __builtin_amdgcn_sched_barrier(0);  // the reads go out before the products that they run beside
                multiply(0);
                wait_copies<COPIES *(STAGES - 2)>();  // step t + 1 is there, and every wave has read step t
                read(t + 1, 0);
                copy(t + STAGES);
                __builtin_amdgcn_sched_barrier(0);
                multiply(1);
            }
            for (; t < n; ++t) {
                read(t, 1);
                multiply(0);
                wait_copies<0>();
                if (t + 1 < n) read(t + 1, 0);
                multiply(1);
            }
        }
    }
    if (tail < t1) {  // through registers, two steps ahead, and two buffers
        i32x4 v[ALIGNED ? 1 : 2][COPIES];
        auto one = [&](int t, i32x4 (&now)[COPIES]) {
            store(t, now);
            if (!ALIGNED && t + 2 < t1) load(t + 2, now);
            wait_copies<63>();
            read(t & 1, 0);
            read(t & 1, 1);
            multiply(0);
            multiply(1);
        };
        wait_copies<0>();  // the ring is through
        load(tail, v[0]);
        if constexpr (ALIGNED) {
            one(tail, v[0]);  // the last step, which is not whole
        } else {
            if (tail + 1 < t1) load(tail + 1, v[1]);
            for (int t = tail; t < t1; t += 2) {
                one(t, v[0]);
                if (t + 1 < t1) one(t + 1, v[1]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int i = i0 + wm + t * 16 + lane % 16, j = j0 + wn + lane / 16 * (4 * TN);
        constexpr int N = TN * 4 < 8 ? TN * 4 : 8;
#pragma unroll
        for (int h = 0; h < TN * 4 / N; ++h) {
            int sum[N];
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = acc[h * (N / 4) + e / 4][t][e % 4];
            if (g.splits == 1) {
                store_row<T, N>(g, i, j + h * N, sum);
            } else if (i < g.m) {
                int *to = g.part + (int64_t(split) * g.m + i) * g.n + j + h * N;
                if (j + (h + 1) * N <= g.n) {
                    __builtin_memcpy(to, sum, sizeof sum);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (j + h * N + e < g.n) to[e] = sum[e];
                }
            }
        }
    }
}

// Adds the splits' integer sums and scales them: four columns of a row to a thread (64 x 4096, 4 splits: 4.4 us).
template <typename T>
__global__ __launch_bounds__(256) void gemm_join_kernel(GemmArgs g)
{
    const int quads = (g.n + 3) / 4;
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int i = int(id / quads), j = int(id % quads) * 4;
    if (i >= g.m) return;
    int sum[4] = {};
    for (int s = 0; s < g.splits; ++s) {
        const int *from = g.part + (int64_t(s) * g.m + i) * g.n + j;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < g.n) sum[e] += from[e];
    }
    store_row<T, 4>(g, i, j, sum);
}

// Up to 16 tokens: bound by reading the weights, which go straight from memory into the registers that the matrix
// instructions take.  Sixteen channels to a workgroup, whose WAVES waves split k (a wave takes 256 bytes of each
// row at a time, a load of it 64, two turns' loads under way together) and add their sums in LDS.
// 1 x 16384 x 4096: 16 us, 4.2 TB/s of weights; 16 x 16384 x 4096: 22 us; 1 x 2560 x 2048: 3.7 us, of which most is a
// launch.
template <typename T, int WAVES, bool ALIGNED>
__global__ __launch_bounds__(64 * WAVES) void gemm_few_kernel(GemmArgs g)
{
    __shared__ i32x4 lds[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * 16, r = lane % 16, at = lane / 16 * 16;
    const int8_t *b = g.b + (j0 + r < g.n ? j0 + r : g.n - 1) * g.ldb;
    const int8_t *a = g.a + (r < g.m ? r : g.m - 1) * g.lda;
    i32x4 acc[2] = {};
    int k = wave * 256;
    if constexpr (ALIGNED) {
        auto step = [&](auto parts) {
            constexpr int N = decltype(parts)::value;
            i32x4 fb[N][4], fa[N][4];
#pragma unroll
            for (int h = 0; h < N; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    fb[h][q] = *reinterpret_cast<const i32x4 *>(b + k + h * (WAVES * 256) + at + q * 64);
                    fa[h][q] = *reinterpret_cast<const i32x4 *>(a + k + h * (WAVES * 256) + at + q * 64);
                }
#pragma unroll
            for (int h = 0; h < N; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    acc[q & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[h][q], fa[h][q], acc[q & 1], 0, 0, 0);
            k += N * WAVES * 256;
        };
        while (k + WAVES * 256 + 256 <= g.k) step(std::integral_constant<int, 2>());
        if (k + 256 <= g.k) step(std::integral_constant<int, 1>());
    } else {
        const int sa = int(uintptr_t(a + at) & 3), sb = int(uintptr_t(b + at) & 3);
        for (; k + 256 <= g.k; k += WAVES * 256) {
            Words wb[4], wa[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                wb[q].load(b + k + at + q * 64);
                wa[q].load(a + k + at + q * 64);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc[q & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wb[q].bytes(sb), wa[q].bytes(sa), acc[q & 1], 0, 0, 0);
        }
    }
    if (k < g.k) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int left = g.k - k - at - q * 64;
            const i32x4 fb = load16(b + k + at + q * 64, left), fa = load16(a + k + at + q * 64, left);
            acc[q & 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, fa, acc[q & 1], 0, 0, 0);
        }
    }
    lds[wave][lane] = acc[0] + acc[1];
    __syncthreads();
    if (wave > 0) return;
    i32x4 v = lds[0][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += lds[w][lane];
    const int sum[4] = {v[0], v[1], v[2], v[3]};
    store_row<T, 4>(g, r, j0 + lane / 16 * 4, sum);  // column r of the result is token r
}

// Copies the rows of both operands, k bytes each, to rows of `ld` (k rounded up to 16), filled up with zeros: first a's
// m rows, then b's n.  16 bytes to a thread (17 MB: 12 us).
__global__ __launch_bounds__(256) void gemm_pack_kernel(GemmArgs g, int8_t *to, int ld)
{
    const int pieces = ld / 16;
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x, row = id / pieces;
    if (row >= g.m + g.n) return;
    const int at = int(id - row * pieces) * 16;
    const int8_t *from = row < g.m ? g.a + row * g.lda : g.b + (row - g.m) * g.ldb;
    *reinterpret_cast<i32x4 *>(to + row * ld + at) = load16(from + at, g.k - at);
}

// Which kernel a product takes.  Up to 16 tokens: the weights straight into registers.  Otherwise tiles, the
// largest that still give every compute unit one; 64 x 64 ones split k where there are too few.
// Larger tiles take rows at multiples of 16 bytes only: with k no multiple of 16, operands that lie otherwise are
// copied first, both, with zeros up to a multiple (4096 x 4096 x 4095: 166 us through
// registers, 88 so).
enum Kind { kFew, kSmall, kMedium, kLarge };

struct GemmPlan {
    Kind kind;
    int tiles_m, tiles_n, splits, per;
    size_t bytes;       // of partial sums
    bool pack;          // operands are copied if one is not aligned
    size_t pack_bytes;  // of both operands
};

// aligned: both operands' rows begin at multiples of 16 bytes.
GemmPlan plan_gemm(int64_t m, int64_t n, int64_t k, bool aligned)
{
    GemmPlan p{kFew, 0, 0, 1, 0, 0, false, 0};
    if (m <= 16 || n == 0) return p;
    const auto tiles = [&](int bm, int bn) { return ceil_div(m, bm) * ceil_div(n, bn); };
    const int64_t steps = ceil_div(k, kStep);
    int side = 64;
    p.kind = kSmall;
    p.pack = k % 16 != 0 && tiles(128, 128) >= 192;
    if (p.pack) p.pack_bytes = size_t(m + n) * size_t(ceil_div(k, 16) * 16);
    aligned = aligned || p.pack;
    if (aligned && tiles(256, 256) >= 224) {
        side = 256;
        p.kind = kLarge;
    } else if (aligned && tiles(128, 128) >= 192) {
        side = 128;
        p.kind = kMedium;
    }
    p.tiles_m = int(ceil_div(m, side));
    p.tiles_n = int(ceil_div(n, side));
    int64_t splits = 1;
    if (p.kind == kSmall) {
        // some 256 workgroups, of 4 steps (512 bytes of k) at least; up to 512, two to a compute unit, where each still
        // has 32 (1198 x 387 x 15466: 133 workgroups 66 us, 399 43 us; with 16 steps each 256 x 4096 x 4096 is slower,
        // 21 us with 512 workgroups against 13 with 256)
        const int64_t few = 256 / tiles(64, 64) < steps / 4 ? 256 / tiles(64, 64) : steps / 4;
        const int64_t more = 512 / tiles(64, 64) < steps / 32 ? 512 / tiles(64, 64) : steps / 32;
        splits = few > more ? few : more;
        if (splits > 16) splits = 16;
        if (splits < 1) splits = 1;
    }
    p.per = int(ceil_div(steps, splits));
    p.splits = p.per > 0 ? int(ceil_div(steps, p.per)) : 1;
    if (p.splits > 1) p.bytes = size_t(p.splits) * size_t(m) * size_t(n) * sizeof(int);
    return p;
}

template <typename T, int BM, int BN, int WM, int WN, int STAGES>
int launch_tile(const GemmArgs &g, bool aligned, hipStream_t st)
{
    constexpr int kLds = STAGES * (BM + BN) * kStep;
    const dim3 grid(static_cast<unsigned>(g.tiles_m * g.tiles_n * g.splits));
    if (aligned) {
        static const hipError_t asked =
            hipFuncSetAttribute(reinterpret_cast<const void *>(gemm_tile_kernel<T, BM, BN, WM, WN, STAGES, true>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (asked != hipSuccess) return AMSIM_ERR_HIP;
        hipLaunchKernelGGL((gemm_tile_kernel<T, BM, BN, WM, WN, STAGES, true>), grid, dim3(64 * WM * WN), kLds, st, g);
    } else if constexpr (BM <= 64) {
        hipLaunchKernelGGL((gemm_tile_kernel<T, BM, BN, WM, WN, STAGES, false>), grid, dim3(64 * WM * WN), 2 * kLds / STAGES, st,
                           g);
    }
    return AMSIM_OK;
}

template <typename T>
int launch_gemm(const GemmPlan &p, const GemmArgs &g, bool aligned, hipStream_t st)
{
    int rc = AMSIM_OK;
    switch (p.kind) {
    case kFew:
        if (aligned)
            hipLaunchKernelGGL((gemm_few_kernel<T, 8, true>), dim3(static_cast<unsigned>(ceil_div(g.n, 16))), dim3(512), 0, st, g);
        else
            hipLaunchKernelGGL((gemm_few_kernel<T, 8, false>), dim3(static_cast<unsigned>(ceil_div(g.n, 16))), dim3(512), 0, st, g);
        break;
    case kSmall: rc = launch_tile<T, 64, 64, 2, 2, 4>(g, aligned, st); break;
    case kMedium: rc = launch_tile<T, 128, 128, 2, 2, 2>(g, aligned, st); break;
    case kLarge: rc = launch_tile<T, 256, 256, 2, 4, 2>(g, aligned, st); break;
    }
    if (rc != AMSIM_OK) return rc;
    if (p.splits > 1)
        hipLaunchKernelGGL((gemm_join_kernel<T>), dim3(static_cast<unsigned>(ceil_div(int64_t(g.m) * ((g.n + 3) / 4), 256))),
                           dim3(256), 0, st, g);
    return launch_status();
}

}  // namespace

extern "C" {

int amsim_gemm_i8_workspace_size(int64_t m, int64_t n, int64_t k, size_t *bytes)
{
    if (!bytes || m < 0 || n < 0 || k < 0) return AMSIM_ERR_INVALID_ARG;
    const int64_t lim = int64_t(1) << 21;
    if (m >= lim || n >= lim || k > kMaxK) return AMSIM_ERR_UNSUPPORTED;
    const GemmPlan any = plan_gemm(m, n, k, false), aligned = plan_gemm(m, n, k, true);
    *bytes = m == 0 || n == 0 ? 0 : (any.bytes > aligned.bytes ? any.bytes : aligned.bytes) + any.pack_bytes;
    return AMSIM_OK;
}

int amsim_gemm_i8(int64_t m, int64_t n, int64_t k, const int8_t *a, int64_t lda, const float *a_scale,
                  const int8_t *b, int64_t ldb, const float *b_scale, const float *bias, int out_dtype, void *c,
                  int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_type(out_dtype)) return AMSIM_ERR_INVALID_ARG;
    size_t need = 0;
    const int rc = amsim_gemm_i8_workspace_size(m, n, k, &need);
    if (rc != AMSIM_OK) return rc;
    if (m == 0 || n == 0) return AMSIM_OK;
    if (!a_scale || !b_scale || !c || ldc < n) return AMSIM_ERR_INVALID_ARG;
    if (k > 0 && (!a || !b || lda < k || ldb < k)) return AMSIM_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need)) return AMSIM_ERR_WORKSPACE;
    if (uintptr_t(workspace) & 15) return AMSIM_ERR_INVALID_ARG;
    // offsets inside a tile are 32-bit numbers there
    const auto whole = [](const void *p, int64_t ld) { return ((uintptr_t(p) | uintptr_t(ld)) & 15) == 0 && ld < (1 << 23); };
    bool aligned = whole(a, lda) && whole(b, ldb);
    const GemmPlan p = plan_gemm(m, n, k, aligned);
    // a launch takes fewer than 2^32 threads (small tiles of 137 GB of results, copies of 64 GB of operands do not fit;
    // larger tiles reach it with results that no memory holds)
    const int64_t threads = int64_t(p.tiles_m) * p.tiles_n * p.splits * (p.kind == kLarge ? 512 : 256);
    const int64_t pieces = p.pack && !aligned ? (m + n) * ceil_div(k, 16) : 0;
    if (threads >= int64_t(1) << 32 || pieces >= int64_t(1) << 32) return AMSIM_ERR_UNSUPPORTED;
    GemmArgs g{a, b, a_scale, b_scale, bias, c, static_cast<int *>(workspace), lda, ldb, ldc, int(m), int(n),
               int(k), p.tiles_m, p.tiles_n, p.splits, p.per};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.pack && !aligned) {  // such plans split nothing: the workspace is the copies'
        const int64_t ld = ceil_div(k, 16) * 16;
        int8_t *to = static_cast<int8_t *>(workspace);
        hipLaunchKernelGGL(gemm_pack_kernel, dim3(static_cast<unsigned>(ceil_div((m + n) * (ld / 16), 256))), dim3(256), 0, st, g,
                           to, int(ld));
        g.a = to;
        g.b = to + m * ld;
        g.lda = g.ldb = ld;
        g.k = int(ld);
        aligned = true;
    }
    return with_type(out_dtype, [&](auto t) { return launch_gemm<decltype(t)>(p, g, aligned, st); });
}

}  // extern "C"
