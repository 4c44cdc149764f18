// Low-rank adapters of many requests beside a shared layer: out[m] = fp16(y[m] + scale[a] B[a] (A[a] x[m])), a = ids[m].
//
// Two kernels over blocks of 16 rows.  The first multiplies a block's rows with the A of every adapter that occurs among them (v_mfma_f32_16x16x32_f16; an
// adapter's result is kept for its own rows only, so that nothing of one adapter, infinities included, reaches another one's rows) and leaves
// the sums over a part of K in the workspace; the second adds the parts up, multiplies with B and adds the shared layer's output.
// The low-rank values are rounded to binary16 between the two (relative to their row's largest: 2^-12 of what the adapter adds).
#include "qfc_internal.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct AdapterArgs {
    const _Float16 *x, *a, *b, *y;  // [M, K], [count, rank, K], [count, N, rank], [M, N]
    const float *scale;             // [count]
    const int *ids;                 // [M]
    float *low;                     // [parts, 16 blocks, rank]
    _Float16 *out;
    int M, K, N, rank, count, parts, part_k, rows;  // rows: M rounded up to 16
};

// Smallest id above `last` among the 16 rows of a block (id in lane m of each quarter), INT32_MAX if there is none
__device__ __forceinline__ int next_id(int id, int last) {
    int next = id > last ? id : INT32_MAX;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) next = min(next, __shfl_xor(next, off, 64));
    return __builtin_amdgcn_readfirstlane(next);
}
__device__ __forceinline__ int row_id(const AdapterArgs &a, int row) {
    const int id = row < a.M ? a.ids[row] : -1;
    return id >= 0 && id < a.count ? id : -1;
}

// grid = (blocks of 16 rows, parts of K); the four wavefronts of a workgroup take the part's pieces of 32 k in turn.  RT: tiles of 16 low-rank values.
template <int RT>
__global__ __launch_bounds__(256) void adapters_shrink_kernel(AdapterArgs a) {
    __shared__ float sums[4][RT][64][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, r = lane >> 4;
    const int row0 = (int)blockIdx.x * 16, k0 = (int)blockIdx.y * a.part_k, k1 = min(k0 + a.part_k, a.K);
    const int id = row_id(a, row0 + m);
    int ids4[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ids4[i] = __shfl(id, 4 * r + i, 64);
    const _Float16 *x = a.x + (size_t)min(row0 + m, a.M - 1) * a.K + 8 * r;
    v4f kept[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) kept[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int one = next_id(id, -1); one != INT32_MAX; one = next_id(id, one)) {
        v4f acc[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = k0 + 32 * wave; k < k1; k += 128) {
            const h8 xv = *reinterpret_cast<const h8 *>(x + k);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                h8 w = {};
                if (16 * t + m < a.rank) w = *reinterpret_cast<const h8 *>(a.a + ((size_t)one * a.rank + 16 * t + m) * a.K + k + 8 * r);
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv, w, acc[t], 0, 0, 0);
            }
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) kept[t][i] = ids4[i] == one ? acc[t][i] : kept[t][i];
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<v4f *>(sums[wave][t][lane]) = kept[t];
    __syncthreads();
    // lane (m, r), element i: row 4 r + i, low-rank value 16 t + m
    for (int t = wave; t < RT; t += 4) {
        if (16 * t + m >= a.rank) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = (sums[0][t][lane][i] + sums[1][t][lane][i]) + (sums[2][t][lane][i] + sums[3][t][lane][i]);
            a.low[((size_t)blockIdx.y * a.rows + row0 + 4 * r + i) * a.rank + 16 * t + m] = v;
        }
    }
}

// grid = (blocks of 16 rows, pieces of 128 columns): a wavefront takes 32 columns.  The low-rank values are the second operand (rows as columns of the result), so that a lane
// ends up with 8 consecutive columns of a row: row i of tile t of B is column 8 (i / 4) + 4 t + i % 4.  KT: steps of 32 low-rank values.
template <int KT>
__global__ __launch_bounds__(256) void adapters_expand_kernel(AdapterArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, r = lane >> 4;
    const int row = (int)blockIdx.x * 16 + m, n0 = ((int)blockIdx.y * 4 + wave) * 32;
    if (n0 >= a.N) return;
    const int id = row_id(a, row);
    // lane (m, r): low-rank values 32 t + 8 r .. + 7 of its row, the row's largest scaled to 2^13 .. 2^14
    float low[KT][8], top = 0.0f;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) low[t][e] = 0.0f;
    for (int p = 0; p < a.parts; ++p) {
        const float *src = a.low + ((size_t)p * a.rows + row) * a.rank;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            if (32 * t + 8 * r < a.rank) {
                const v4f l0 = *reinterpret_cast<const v4f *>(src + 32 * t + 8 * r), l1 = *reinterpret_cast<const v4f *>(src + 32 * t + 8 * r + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    low[t][e] += l0[e];
                    low[t][4 + e] += l1[e];
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(low[t][e]));
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const int up = top > 0.0f && top < INFINITY ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
    h8 v[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[t][e] = (_Float16)__builtin_amdgcn_ldexpf(low[t][e], up);
    const float scale = id >= 0 ? a.scale[id] : 0.0f;

    v4f kept[2] = {v4f{0.0f, 0.0f, 0.0f, 0.0f}, v4f{0.0f, 0.0f, 0.0f, 0.0f}};
    for (int one = next_id(id, -1); one != INT32_MAX; one = next_id(id, one)) {
        const bool own = id == one;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int n = n0 + 8 * (m >> 2) + 4 * t + (m & 3);
            v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                h8 w = {};
                if (n < a.N && 32 * k + 8 * r < a.rank) w = *reinterpret_cast<const h8 *>(a.b + ((size_t)one * a.N + n) * a.rank + 32 * k + 8 * r);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, v[k], acc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) kept[t][i] = own ? acc[i] : kept[t][i];
        }
    }
    if (row >= a.M) return;
    const int n = n0 + 8 * r;
    const size_t at = (size_t)row * a.N + n;
    float add[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) add[e] = __builtin_amdgcn_ldexpf(kept[e >> 2][e & 3], -up) * scale;
    if (a.N % 8 == 0) {
        if (n >= a.N) return;
        h8 y = *reinterpret_cast<const h8 *>(a.y + at);
        if (id >= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (_Float16)((float)y[e] + add[e]);
        }
        *reinterpret_cast<h8 *>(a.out + at) = y;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (n + e >= a.N) break;
        const _Float16 y = a.y[at + e];
        a.out[at + e] = id >= 0 ? (_Float16)((float)y + add[e]) : y;
    }
}

}  // namespace

AdapterPlan plan_adapters(int M, int K, int num_cus) {
    AdapterPlan p;
    p.rows = round_up(M, 16);
    const int blocks = p.rows / 16, pieces = (K + 127) / 128;
    int parts = (2 * num_cus + blocks - 1) / blocks;
    if (parts > 16) parts = 16;
    if (parts > pieces) parts = pieces;
    if (parts < 1) parts = 1;
    p.part_k = (pieces + parts - 1) / parts * 128;
    p.parts = (K + p.part_k - 1) / p.part_k;
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
    g.parts = p.parts, g.part_k = p.part_k, g.rows = p.rows;
    const dim3 shrink((unsigned)(p.rows / 16), (unsigned)p.parts), expand((unsigned)(p.rows / 16), (unsigned)((N + 127) / 128));
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
        adapters_expand_kernel<1><<<expand, 256, 0, st>>>(g);
    else if (rank <= 64)
        adapters_expand_kernel<2><<<expand, 256, 0, st>>>(g);
    else
        adapters_expand_kernel<4><<<expand, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace qfc
