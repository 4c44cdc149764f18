// Low-rank adapters of many requests beside a shared layer: out[m] = fp16(y[m] + scale[a] B[a] (A[a] x[m])), a = ids[m].
//
// Two kernels.  The first multiplies blocks of 16 rows with the A of every adapter that occurs among them (v_mfma_f32_16x16x32_f16) and leaves
// the sums over a part of K in the workspace, in 32 bits; the second adds the parts up, multiplies with B and adds the shared layer's output.  An adapter's results are kept for its
// own rows only, so that nothing of one adapter, infinities included, reaches another one's rows.  Where every row has an adapter of its own (a decode step), the adapters of a
// block of rows are dealt to several workgroups.
// The low-rank values are rounded to binary16 between the two, scaled by a power of two to their row's largest (2^-11 of a value, 2^-38 of the largest), for the matrix product;
// the output is rounded once.  Bound: memory (A and B of the adapters in use, x, y and out), for few rows the latency of two launches.
#include "qfc_internal.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct AdapterArgs {
    const _Float16 *x, *a, *b, *y;  // [M, K], [count, rank, K], [count, N, rank], [M, N]
    const float *scale;             // [count]
    const int *ids;                 // [M]
    float *low;                     // [parts, rows, rank]
    _Float16 *out;
    int M, K, N, rank, count, parts, part_k, rows, dealt, tiles;  // rows: M rounded up; dealt: workgroups that share a block's adapters; tiles: of 32 columns per wavefront
};

// Adapter of row row0 + lane of a block of ROWS, -1 for none
template <int ROWS>
__device__ __forceinline__ int row_id(const AdapterArgs &a, int row0, int lane) {
    const int id = lane < ROWS && row0 + lane < a.M ? a.ids[row0 + lane] : -1;
    return id >= 0 && id < a.count ? id : -1;
}
// f(adapter, its rows' bits) for the adapters of the block that are this workgroup's, in the order of their first rows
template <class F>
__device__ __forceinline__ void for_adapters(int id, int mine, int dealt, const F &f) {
    uint64_t left = __ballot(id >= 0);
    for (int turn = 0; left; turn = turn + 1 == dealt ? 0 : turn + 1) {
        const int one = __builtin_amdgcn_readlane(id, __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)left) - 1));
        const uint64_t rows = __ballot(id == one);
        left &= ~rows;
        if (turn == mine) f(one, rows);
    }
}

// grid = (blocks of 16 rows, parts of K, workgroups that share a block's adapters); the four wavefronts of a workgroup take the part's pieces of 64 k in turn.  RT: tiles of 16
// low-rank values.  One row of 4096 values 2.7 us, 64 rows of 40 adapters of rank 16 4.8 us, 2048 rows of 5 adapters of rank 64 23 us (20 MB, each block of rows reads its adapters again
// from L2).
template <int RT>
__global__ __launch_bounds__(256) void adapters_shrink_kernel(AdapterArgs a) {
    __shared__ float sums[4][RT][64][4];
    constexpr int U = RT <= 4 ? 4 : 2;  // pieces on their way at once
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, r = lane >> 4;
    const int row0 = (int)blockIdx.x * 16, k0 = (int)blockIdx.y * a.part_k, k1 = min(k0 + a.part_k, a.K);
    const int id = row_id<16>(a, row0, lane);
    const _Float16 *x = a.x + (size_t)min(row0 + m, a.M - 1) * a.K + 8 * r;
    v4f kept[RT];
    uint64_t done = 0;
#pragma unroll
    for (int t = 0; t < RT; ++t) kept[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for_adapters(id, blockIdx.z, a.dealt, [&](int one, uint64_t rows) __attribute__((always_inline)) {
        done |= rows;
        const _Float16 *w = a.a + (size_t)one * a.rank * a.K + (size_t)m * a.K + 8 * r;
        v4f acc[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = k0 + 64 * wave; k < k1; k += 128 * U) {
            h8 xv[U], wv[U][RT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const h8 zero = {};
                const int ku = k + 32 * (u & 1) + 256 * (u >> 1);
                const bool there = ku < k1;
                xv[u] = there ? *reinterpret_cast<const h8 *>(x + ku) : zero;
#pragma unroll
                for (int t = 0; t < RT; ++t) wv[u][t] = there && 16 * t + m < a.rank ? *reinterpret_cast<const h8 *>(w + (size_t)16 * t * a.K + ku) : zero;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[u], wv[u][t], acc[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) kept[t][i] = rows >> (4 * r + i) & 1 ? acc[t][i] : kept[t][i];
    });
    if (!done) return;  // (the same in all four wavefronts)
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<v4f *>(sums[wave][t][lane]) = kept[t];
    __syncthreads();
    // lane (m, r), element i: row 4 r + i, low-rank value 16 t + m
    for (int t = wave; t < RT; t += 4) {
        if (16 * t + m >= a.rank) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = (sums[0][t][lane][i] + sums[1][t][lane][i]) + (sums[2][t][lane][i] + sums[3][t][lane][i]);
            if (done >> (4 * r + i) & 1) a.low[((size_t)blockIdx.y * a.rows + row0 + 4 * r + i) * a.rank + 16 * t + m] = v;
        }
    }
}

// grid = (blocks of 16 MT rows x pieces of 128 `tiles` columns, workgroups that share a block's adapters): the blocks of a piece side by side on one XCD, whose L2 then
// has the piece of B.  The workgroup adds up its rows' low-rank values once, into LDS; then a
// wavefront takes 32 columns at a time, each of B's tiles for all of the block's rows.  The low-rank values are the second operand (rows as columns of the result), so that a lane
// ends up with 8 consecutive columns of a row: row i of tile t of B is column 8 (i / 4) + 4 t + i % 4.  KT: steps of 32 low-rank values.
// One row of 6144 columns 4.8 us, 64 rows of 40 adapters and 4096 columns 8.0 us, both latency; 2048 rows of 28672 columns 83 us for 252 MB (3.0 TB/s; the same loads and stores of y and
// out without the products take 33 us: what is left is waiting, with two wavefronts on a SIMD, for loads and stores that share a counter).
template <int KT, int MT>
__global__ __launch_bounds__(256) void adapters_expand_kernel(AdapterArgs a) {
    constexpr int ROWS = 16 * MT, PITCH = 32 * KT + 8;
    __shared__ _Float16 low[ROWS][PITCH];
    __shared__ uint32_t top[ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, r = lane >> 4;
    const int blocks = (a.M + ROWS - 1) / ROWS, turn = (int)blockIdx.x / 8;
    const int piece = (int)blockIdx.x % 8 + 8 * (turn / blocks), row0 = turn % blocks * ROWS;
    if (piece * a.tiles * 128 >= a.N) return;
    const int id = row_id<ROWS>(a, row0, lane);
    uint64_t own = 0;
    for_adapters(id, blockIdx.y, a.dealt, [&](int, uint64_t rows) __attribute__((always_inline)) { own |= rows; });
    // rows without an adapter: the first of the workgroups copies them
    const uint64_t plain = blockIdx.y == 0 ? __ballot(id < 0 && lane < ROWS && row0 + lane < a.M) : 0;
    if (!(own | plain)) return;

    // What does not depend on the low-rank values is requested before they are read: the first columns' outputs and the first adapter's tile
    auto columns = [&](int c) __attribute__((always_inline)) { return ((piece * a.tiles + c) * 4 + wave) * 32; };
    auto load_y = [&](int c, h8 (&y)[MT]) __attribute__((always_inline)) {
        const int n = columns(c) + 8 * r;
        if (a.N % 8 != 0 || n >= a.N || c >= a.tiles) return;
#pragma unroll
        for (int t = 0; t < MT; ++t)
            if ((own | plain) >> (16 * t + m) & 1) y[t] = *reinterpret_cast<const h8 *>(a.y + (size_t)(row0 + 16 * t + m) * a.N + n);
    };
    auto load_w = [&](int c, int one, h8 (&w)[2][KT]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int col = columns(c) + 8 * (m >> 2) + 4 * u + (m & 3);
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                const h8 zero = {};
                w[u][k] = col < a.N && 32 * k + 8 * r < a.rank ? *reinterpret_cast<const h8 *>(a.b + ((size_t)one * a.N + col) * a.rank + 32 * k + 8 * r) : zero;
            }
        }
    };
    const int first = own ? __builtin_amdgcn_readlane(id, __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)own) - 1)) : -1;
    h8 y[MT], w0[2][KT];
    load_y(0, y);
    if (first >= 0) load_w(0, first, w0);

    if (own) {
        constexpr int MOST = ROWS * KT * 4 / 256 > 0 ? ROWS * KT * 4 / 256 : 1;  // octets per thread
        const int octets = a.rank / 8;
        float v[MOST][8];
        if (threadIdx.x < ROWS) top[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < MOST; ++q) {
            const int e = threadIdx.x + 256 * q, row = e / octets, o = e % octets;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[q][i] = 0.0f;
            if (row < ROWS && (own >> row & 1)) {
                const float *src = a.low + (size_t)(row0 + row) * a.rank + 8 * o;
                for (int p0 = 0; p0 < a.parts; p0 += 8) {  // (eight parts on their way at once; those behind the last read it again and are left out)
                    v4f l[8][2];
#pragma unroll
                    for (int p = 0; p < 8; ++p) {
                        const float *part = src + (size_t)min(p0 + p, a.parts - 1) * a.rows * a.rank;
                        l[p][0] = *reinterpret_cast<const v4f *>(part);
                        l[p][1] = *reinterpret_cast<const v4f *>(part + 4);
                    }
#pragma unroll
                    for (int p = 0; p < 8; ++p)
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[q][i] = p0 + p < a.parts ? v[q][i] + l[p][i >> 2][i & 3] : v[q][i];
                }
                float big = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(v[q][i]));
                atomicMax(&top[row], __float_as_uint(big));  // (a maximum: whatever the order)
            }
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < MOST; ++q) {
            const int e = threadIdx.x + 256 * q, row = e / octets, o = e % octets;
            if (row >= ROWS) continue;
            const float big = __uint_as_float(top[row]);
            const int up = big > 0.0f && big < INFINITY ? 14 - __builtin_amdgcn_frexp_expf(big) : 0;  // the row's largest to 2^13 .. 2^14
            h8 x;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (_Float16)__builtin_amdgcn_ldexpf(v[q][i], up);
            *reinterpret_cast<h8 *>(&low[row][8 * o]) = x;
        }
        for (int e = threadIdx.x; e < ROWS * (4 * KT - octets); e += 256) {
            const h8 zero = {};
            *reinterpret_cast<h8 *>(&low[e / (4 * KT - octets)][8 * (octets + e % (4 * KT - octets))]) = zero;
        }
        __syncthreads();
    }
    auto low_at = [&](int t, int k) __attribute__((always_inline)) { return *reinterpret_cast<const h8 *>(&low[16 * t + m][32 * k + 8 * r]); };  // (in LDS: registers are for what is on its way)
    float back[MT];  // the scale and the power of two taken back
    bool real[MT], has[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int row = 16 * t + m;
        has[t] = own >> row & 1;
        real[t] = (own | plain) >> row & 1;
        const float big = own ? __uint_as_float(top[row]) : 0.0f;
        const int up = big > 0.0f && big < INFINITY ? 14 - __builtin_amdgcn_frexp_expf(big) : 0;
        const int of_row = __shfl(id, row, 64);
        back[t] = has[t] ? __builtin_amdgcn_ldexpf(a.scale[of_row], -up) : 0.0f;
    }
    int c = 0;
    // Every row there and this workgroup's, whole tiles: no branches but the loop over the adapters, so that the loads of the next columns are not waited for.
    if (own && (own | plain) == (ROWS == 64 ? ~0ull : (1ull << ROWS) - 1) && a.N % 8 == 0) {
        const _Float16 *yp[MT];
        _Float16 *op[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            yp[t] = a.y + (size_t)(row0 + 16 * t + m) * a.N + columns(0) + 8 * r;
            op[t] = a.out + (size_t)(row0 + 16 * t + m) * a.N + columns(0) + 8 * r;
        }
        const int whole = a.N > columns(0) ? min(a.tiles, ((a.N - columns(0)) / 32 + 3) / 4) : 0;  // tiles of 32 columns of this wavefront, four apart
        const uint64_t firsts = __ballot(id == first), others = own & ~firsts;
        // (every address is one to read from, and what is not wanted is dropped: no branches around the loads)
        const _Float16 *wp[2][KT];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < KT; ++k) wp[u][k] = a.b + ((size_t)columns(0) + 8 * (m >> 2) + 4 * u + (m & 3)) * a.rank + min(32 * k + 8 * r, a.rank - 8);
        auto load_whole = [&](int tile, int one, h8 (&w)[2][KT]) __attribute__((always_inline)) {
            const size_t off = ((size_t)one * a.N + tile * 128) * a.rank;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < KT; ++k) w[u][k] = *reinterpret_cast<const h8 *>(wp[u][k] + off);
        };
        auto cut = [&](h8 (&w)[2][KT]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    const h8 zero = {};
                    w[u][k] = 32 * k + 8 * r < a.rank ? w[u][k] : zero;
                }
        };
        auto work = [&](h8 (&yc)[MT], h8 (&wc)[2][KT], h8 (&yn)[MT], h8 (&wn)[2][KT]) __attribute__((always_inline)) {
            const int next = min(c + 1, whole - 1) * 128;
#pragma unroll
            for (int t = 0; t < MT; ++t) yn[t] = *reinterpret_cast<const h8 *>(yp[t] + next);
            load_whole(min(c + 1, whole - 1), first, wn);
            cut(wc);
            v4f kept[MT][2];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                kept[t][0] = kept[t][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int u = 0; u < 2; ++u) kept[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wc[u][k], low_at(t, k), kept[t][u], 0, 0, 0);
            }
            for (uint64_t left = others; left;) {
                const int one = __builtin_amdgcn_readlane(id, __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)left) - 1));
                const uint64_t rows = __ballot(id == one);
                left &= ~rows;
                h8 w[2][KT];
                load_whole(c, one, w);
                cut(w);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int k = 0; k < KT; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[u][k], low_at(t, k), acc, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) kept[t][u][i] = rows >> (16 * t + m) & 1 ? acc[i] : kept[t][u][i];
                    }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                h8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = has[t] ? (_Float16)((float)yc[t][e] + kept[t][e >> 2][e & 3] * back[t]) : yc[t][e];
                *reinterpret_cast<h8 *>(op[t] + c * 128) = o;
            }
            ++c;
        };
        h8 y1[MT], w1[2][KT];
        while (c + 1 < whole) {
            work(y, w0, y1, w1);
            work(y1, w1, y, w0);
        }
        if (c < whole) work(y, w0, y1, w1);
        if (c < a.tiles && columns(c) < a.N) {
            load_y(c, y);
            load_w(c, first, w0);
        }
    }
    for (; c < a.tiles; ++c) {
        const int n0 = columns(c), n = n0 + 8 * r;
        if (n0 >= a.N) return;
        h8 y_next[MT];
        load_y(c + 1, y_next);
        v4f kept[MT][2];
#pragma unroll
        for (int t = 0; t < MT; ++t) kept[t][0] = kept[t][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for_adapters(id, blockIdx.y, a.dealt, [&](int one, uint64_t rows) __attribute__((always_inline)) {
            h8 w[2][KT];
            if (one == first) {  // (requested during the columns before)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int k = 0; k < KT; ++k) w[u][k] = w0[u][k];
                if (c + 1 < a.tiles) load_w(c + 1, first, w0);
            } else {
                load_w(c, one, w);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if (!(rows >> (16 * t) & 0xFFFF)) continue;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < KT; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[u][k], low_at(t, k), acc, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) kept[t][u][i] = rows >> (16 * t + m) & 1 ? acc[i] : kept[t][u][i];
                }
            }
        });
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (!real[t]) continue;
            const size_t at = (size_t)(row0 + 16 * t + m) * a.N + n;
            if (a.N % 8 == 0) {
                if (n >= a.N) continue;
                if (has[t]) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[t][e] = (_Float16)((float)y[t][e] + kept[t][e >> 2][e & 3] * back[t]);
                }
                *reinterpret_cast<h8 *>(a.out + at) = y[t];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (n + e >= a.N) break;
                    const _Float16 old = a.y[at + e];
                    a.out[at + e] = has[t] ? (_Float16)((float)old + kept[t][e >> 2][e & 3] * back[t]) : old;
                }
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) y[t] = y_next[t];
    }
}

template <int KT>
void launch_expand(const AdapterArgs &g, int block_rows, hipStream_t st) {
    const int pieces = (g.N + 128 * g.tiles - 1) / (128 * g.tiles);
    const dim3 grid((unsigned)((g.M + block_rows - 1) / block_rows * round_up(pieces, 8)), (unsigned)g.dealt);
    if (block_rows == 16)
        adapters_expand_kernel<KT, 1><<<grid, 256, 0, st>>>(g);
    else
        adapters_expand_kernel<KT, 4><<<grid, 256, 0, st>>>(g);
}

}  // namespace

AdapterPlan plan_adapters(int M, int K, int N, int num_cus) {
    AdapterPlan p;
    if (num_cus < 1) num_cus = 1;
    p.rows = round_up(M, 64);
    const int blocks = (M + 15) / 16, pieces = (K + 127) / 128, pieces_n = (N + 127) / 128;
    // few rows: up to an adapter for every row, dealt to as many workgroups
    // (64 rows of 40 adapters, 4096 x 4096, 16 / 8 / 4 workgroups per block: 17.1 / 13.3 / 13.8 us; 128 rows 27.5 / 19.3 / 15.4; 16 rows 11.2 / 11.0 / 11.9)
    p.dealt = (int)(4L * num_cus / ((long)blocks * pieces_n));
    if (p.dealt > 16) p.dealt = 16;
    if (p.dealt > M) p.dealt = M;
    if (p.dealt < 1) p.dealt = 1;
    int parts = 2 * num_cus / (blocks * p.dealt);  // (of K, so that few rows reach every compute unit)
    if (parts > 16) parts = 16;
    if (parts > pieces) parts = pieces;
    if (parts < 1) parts = 1;
    p.part_k = (pieces + parts - 1) / parts * 128;
    p.parts = (K + p.part_k - 1) / p.part_k;
    // many rows: blocks of 64 share B's tiles.  (us with 16 / 64, rows of five requests one behind the other: 300 x 28672 21.2 / 19.8, 520 x 6144 17.2 / 16.2, 1000 x 6144 19.4 / 20.6,
    // 2048 x 6144 38 / 29, 1000 x 28672 76 / 58.  Rows in turn with 40 adapters, which the host does not know, would want blocks of 16 up to some 1000 rows: 300 x 4096 30 / 40,
    // 1000 x 6144 77 / 94, 2048 x 6144 183 / 154.)
    // Columns per workgroup so that the card holds all workgroups at once, two to a compute unit (2048 x 28672: 107 us, with four 117 and 112 for blocks of 32; ranks above 64 have
    // registers for one, and take two rounds)
    p.block_rows = M > 256 ? 64 : 16;
    const long works = (long)((M + p.block_rows - 1) / p.block_rows) * pieces_n;
    p.tiles = (int)((works + 2L * num_cus - 1) / (2L * num_cus));
    if (p.tiles > 16) p.tiles = 16;
    if (p.tiles < 1) p.tiles = 1;
    return p;
}

size_t adapters_workspace(const AdapterPlan &p, int rank) { return (size_t)p.parts * p.rows * rank * sizeof(float); }

hipError_t launch_adapters(const void *x, int M, int K, int N, int rank, int count, const void *a, const void *b, const float *scale, const int *ids, const void *y,
                           const AdapterPlan &p, void *workspace, void *out, hipStream_t st) {
    AdapterArgs g;
    g.x = static_cast<const _Float16 *>(x);
    g.a = static_cast<const _Float16 *>(a);
    g.b = static_cast<const _Float16 *>(b);
    g.y = static_cast<const _Float16 *>(y);
    g.scale = scale;
    g.ids = ids;
    g.low = static_cast<float *>(workspace);
    g.out = static_cast<_Float16 *>(out);
    g.M = M, g.K = K, g.N = N, g.rank = rank, g.count = count;
    g.parts = p.parts, g.part_k = p.part_k, g.rows = p.rows, g.dealt = p.dealt, g.tiles = p.tiles;
    const dim3 shrink((unsigned)((M + 15) / 16), (unsigned)p.parts, (unsigned)p.dealt);
    if (rank <= 16)
        adapters_shrink_kernel<1><<<shrink, 256, 0, st>>>(g);
    else if (rank <= 32)
        adapters_shrink_kernel<2><<<shrink, 256, 0, st>>>(g);
    else if (rank <= 64)
        adapters_shrink_kernel<4><<<shrink, 256, 0, st>>>(g);
    else
        adapters_shrink_kernel<8><<<shrink, 256, 0, st>>>(g);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (rank <= 32)
        launch_expand<1>(g, p.block_rows, st);
    else if (rank <= 64)
        launch_expand<2>(g, p.block_rows, st);
    else
        launch_expand<4>(g, p.block_rows, st);
    return hipGetLastError();
}

}  // namespace qfc
