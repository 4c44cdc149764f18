// Attention of the new tokens of a batch of requests over their paged 4-bit cache (layout: paged_q4.h).
//
// With a cached value = offset + step (code - 8), one step and offset per 32 values (group j) of a position's head:
//   q . k = sum_j step_j (q_j . code_j - 8 sum q_j) + sum_j offset_j sum q_j
// so the score product multiplies q with the codes as they are, one v_mfma_f32_16x16x32_f16 per group: a masked nibble is the denormal code * 2^-24, the nibbles in the place 16
// times as high meet queries divided by 16, and the accumulator starts at -8 sum q_j.  The steps multiply the 32-bit result; the offsets come in by one more MFMA, against the sums of
// q in two binary16 parts (2^-22).  For the second product
//   out_d = sum_p (p step_j) (code - 8) + sum_p p offset_j
// P is multiplied with the step in 32 bits and rounded to binary16 once per group; the -8 is taken off with the same rounded values (an MFMA against a
// constant), so that what the rounding leaves is relative to a centred code, and the offsets are again one MFMA, whose last row, ones, gives the sum of P.
// P is taken 2^14 times as large: with steps below 2 every product is below 2^15, and binary16 keeps its 11 bits down to 2^-28.  A
// step of 2 or more (values some 30 apart and more) lowers that factor to 2^2 from there on, for which every step is small enough.
#include "paged_q4.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kMasked = -1.0e30f;
constexpr float kNothingYet = -1.0e25f;  // maximum of a row that has seen no position: above every masked score, below every real one

struct AttnQ4Args {
    const _Float16 *q;  // [tokens, h_q, D]
    _Float16 *out;
    const char *pages;
    Requests req;
    float *ws_o, *ws_ml;  // [batch h_kv, chunks, rows, D] partial outputs, [.., 2] (maximum, sum)
    int h_q, h_kv, g, chunks, chunk_pages, blocks, max_rows;
    float scale;
};

// How many pages the rows row0 .. row0 + 15 of a request see between them, and how many rows there are
struct RowBlock {
    Span span;
    int rows, pages, end;  // end: positions the last row sees
};
__device__ __forceinline__ RowBlock row_block(const AttnQ4Args &a, int b, int row0) {
    RowBlock k;
    k.span = span_of(a.req, b);
    k.rows = k.span.count * a.g;
    k.end = max(0, k.span.positions - k.span.count + min(row0 + 15, k.rows - 1) / a.g + 1);
    k.pages = (k.end + kPage - 1) / kPage;
    return k;
}

// What a wavefront has on its way: DEPTH pages, keys and values each in a place of PART bytes of LDS of its own.
template <int D>
struct Ring {
    static constexpr int kHalf = 40 * D;                      // bytes of a page's keys or values
    static constexpr int PART = (kHalf + 1023) / 1024 * 1024;  // copied in pieces of a KiB
    static constexpr int COPIES = PART / 1024;
    static constexpr int DEPTH = D == 64 ? 3 : 2;
    static constexpr int PITCH = D + 4;  // floats per row of the wavefronts' results
    static constexpr int WAVE = 2 * DEPTH * PART;
    static constexpr int MERGE = 4 * 16 * PITCH * 4;
    static constexpr int LDS = 4 * WAVE > MERGE ? 4 * WAVE : MERGE;
    static constexpr int FLYING = (2 * DEPTH - 1) * COPIES;  // copies behind the ones waited for
    static_assert(LDS <= (D <= 128 ? 80 : 160) * 1024 && FLYING <= 63, "LDS, and the 6-bit counter of outstanding copies");
};

// Workgroup = four wavefronts and up to 16 query rows of a KV head; the wavefronts take the pages of the workgroup's chunk in turn, each with
// copies of its own on the way (no barrier before the end).
template <int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void attn_q4_kernel(AttnQ4Args a) {
    typedef PageLayout<D> L;
    typedef Ring<D> R;
    constexpr int G = L::G, DT = D / 16, W = L::W;
    constexpr int PITCH = R::PITCH;
    extern __shared__ float lds[];  // the rings; then [4][16][PITCH]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, r = lane >> 4;
    int w = blockIdx.x;
    const int chunk = w % a.chunks;
    w /= a.chunks;
    const int group = w % (a.req.batch * a.h_kv), row0 = w / (a.req.batch * a.h_kv) * 16;
    const int b = group / a.h_kv, kv = group % a.h_kv;
    const RowBlock blk = row_block(a, b, row0);
    if (row0 >= blk.rows) return;
    if (chunk > 0 && chunk * a.chunk_pages >= blk.pages) return;
    const int pages = __builtin_amdgcn_readfirstlane(min(blk.pages, (chunk + 1) * a.chunk_pages));
    const int n = blk.span.positions;

    // ---- queries: lane (m, r) holds q[row0 + m][32 j + 8 r .. + 7], scaled by a power of two
    const bool real = row0 + m < blk.rows;
    const int token = real ? (row0 + m) / a.g : 0, head = kv * a.g + (real ? (row0 + m) % a.g : 0);
    const size_t at = ((size_t)(blk.span.first + token) * a.h_q + head) * D;
    const int lim = real ? n - blk.span.count + token + 1 : 0;  // positions the lane's row sees (none where 0 or less)
    h8 qf[G];
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const h8 zero = {};
        qf[j] = real ? *reinterpret_cast<const h8 *>(a.q + at + 32 * j + 8 * r) : zero;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)qf[j][e]));
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    // the largest to 2^13 .. 2^14: what the division by 16 below loses is 2^-24 of it and less
    const int up = top > 0.0f ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
    const float up2 = __builtin_amdgcn_ldexpf(1.0f, up);
    const float to_score = __builtin_amdgcn_ldexpf(a.scale, 24 - up);  // 2^24: the codes' denormals
    float start[G];
    h8 sums = {};
#pragma unroll
    for (int j = 0; j < G; ++j) {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = (float)qf[j][e] * up2;
            s += x;
            qf[j][e] = (_Float16)(e & 2 ? x * 0.0625f : x);  // (values 2, 3, 6, 7 of an octet: the high nibbles of their bytes)
        }
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        start[j] = s * (-8.0f / 16777216.0f);
        const _Float16 hi = (_Float16)(s * 0.0625f), lo = (_Float16)(s * 0.0625f - (float)hi);
        sums[j] = r == 0 ? hi : r == 1 ? lo : (_Float16)0.0f;
    }

    v4f acc[DT], eights[G], rest = {};
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < G; ++j) eights[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float run_max = kNothingYet, lower = 1.0f;  // lower: what P's factor 2^14 has been lowered by
    h8 eight;  // 8 as a denormal code
#pragma unroll
    for (int e = 0; e < 8; ++e) eight[e] = __builtin_bit_cast(_Float16, (uint16_t)8);
    const uint32_t mask_lo = 0x000F000Fu, mask_hi = 0x00F000F0u;

    // ---- copies.  The wavefront's i-th page is first + 4 i; lane i holds the place of page i (of 64 at a time)
    const int first = chunk * a.chunk_pages + wave;
    const int count = first < pages ? (pages - first + 3) / 4 : 0;
    char *const ring = reinterpret_cast<char *>(lds) + wave * R::WAVE;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds + wave * R::WAVE);
    auto places = [&](int i) __attribute__((always_inline)) { return i + lane < count ? page_of(a.req, b, (first + 4 * (i + lane)) * kPage) : -1; };
    int ahead = places(0), now = ahead;  // of the pages that are requested, and of those that are worked on
    auto copy = [&](int i, int slot, int part) __attribute__((always_inline)) {  // part 0: keys, 1: values
        const int page = __builtin_amdgcn_readlane(ahead, i & 63);
        const char *src = a.pages + ((size_t)max(page, 0) * a.h_kv + kv) * L::kBytes + part * R::kHalf;
#pragma unroll
        for (int c = 0; c < R::COPIES; ++c)  // (the last piece's lanes behind the part copy its end again)
            copy16_to_lds(src, (uint32_t)min(c * 1024 + lane * 16, R::kHalf - 16), ring_at + (2 * slot + part) * R::PART + c * 1024);
    };
#pragma unroll
    for (int i = 0; i < R::DEPTH; ++i)
        if (i < count) {
            copy(i, i, 0);
            copy(i, i, 1);
        }
    // The copies of page i are there: as many as ever are behind them while DEPTH pages follow, none later.  In front of a copy into a place all reads of it are done.
    auto wait_for = [&](int i) __attribute__((always_inline)) {
        if (i + R::DEPTH < count)
            wait_copies<R::FLYING>();
        else
            wait_copies<0>();
    };

    for (int i = 0, slot = 0; i < count; ++i, slot = slot + 1 == R::DEPTH ? 0 : slot + 1) {
        const int k0 = (first + 4 * i) * kPage;
        if (i > 0 && (i & 63) == 0) now = places(i);
        if (i + R::DEPTH < count && ((i + R::DEPTH) & 63) == 0) ahead = places(i + R::DEPTH);
        const int page = __builtin_amdgcn_readlane(now, i & 63);
        const char *src = ring + 2 * slot * R::PART;
        wait_for(i);
        const int seen = page >= 0 ? lim - k0 : 0, valid = page >= 0 ? n - k0 : 0;  // of this page, by the lane's row and by anyone

        // ---- scores; lane (m, r), element 4 t + i: position 16 r + 4 t + i, in units of log 2
        float sc[16], bmax = kMasked;
        {
            v4f part[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                h8 off = {};
                if (r < 2) {
#pragma unroll
                    for (int j = 0; j < G; ++j) off[j] = reinterpret_cast<const _Float16 *>(src + L::kOffsetK + (16 * t + m) * G * 2)[j];
                }
                const v4f zero = {};
                part[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, sums, zero, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) part[t][i] *= 1.0f / 1048576.0f;
            }
#pragma unroll
            for (int j = 0; j < G; ++j) {
                h8 st[2];
                st[0] = *reinterpret_cast<const h8 *>(src + L::kStepK + (j * kPage + 16 * r) * 2);
                st[1] = *reinterpret_cast<const h8 *>(src + L::kStepK + (j * kPage + 16 * r + 8) * 2);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t c = *reinterpret_cast<const uint32_t *>(src + L::kCodesK + ((t * (G / W) + j / W) * 64 + lane) * (4 * W) + (j % W) * 4);
                    const u32x4 op = {c & mask_lo, c & mask_hi, (c >> 8) & mask_lo, (c >> 8) & mask_hi};
                    const v4f from = {start[j], start[j], start[j], start[j]};
                    const v4f x = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, op), qf[j], from, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[t][i] = fmaf((float)st[t >> 1][4 * (t & 1) + i], x[i], part[t][i]);
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[4 * t + i] = 16 * r + 4 * t + i < seen ? part[t][i] * to_score : kMasked;
                    bmax = fmaxf(bmax, sc[4 * t + i]);
                }
        }
        wait_copies<63>();  // (the keys have been read)
        if (i + R::DEPTH < count) copy(i + R::DEPTH, slot, 0);
        bmax = fmaxf(bmax, __shfl_xor(bmax, 16, 64));
        bmax = fmaxf(bmax, __shfl_xor(bmax, 32, 64));
        const float new_max = fmaxf(run_max, bmax), corr = __builtin_amdgcn_exp2f(run_max - new_max);
        run_max = new_max;
        h8 pv[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            sc[e] = __builtin_amdgcn_exp2f(sc[e] - new_max + 14.0f);
            pv[e >> 3][e & 7] = (_Float16)sc[e];
        }
        if (__any(corr != 1.0f)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t][i] *= corr;
#pragma unroll
                for (int j = 0; j < G; ++j) eights[j][i] *= corr;
                rest[i] *= corr;
            }
        }

        // ---- second product.  Positions that nobody has may hold anything: their steps and offsets are taken as 0
        wait_for(i);
        src += R::PART - R::kHalf;  // (the layout counts from the page's start)
        h8 step[G][2];
        uint32_t large = 0;
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                h8 s = *reinterpret_cast<const h8 *>(src + L::kStepV + (j * kPage + 16 * r + 8 * u) * 2);
                if (valid < kPage) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] = 16 * r + 8 * u + e < valid ? s[e] : (_Float16)0.0f;
                }
                step[j][u] = s;
                const u32x4 bits = __builtin_bit_cast(u32x4, s);
                large |= bits.x | bits.y | bits.z | bits.w;
            }
        if (lower == 1.0f && __any((large & 0x40004000u) != 0)) {  // a step of 2 or more
            lower = 1.0f / 4096.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t][i] *= lower;
#pragma unroll
                for (int j = 0; j < G; ++j) eights[j][i] *= lower;
            }
        }
        if (lower != 1.0f) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] *= lower;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            h8 off = {};
            if (m < G) {
                off = *reinterpret_cast<const h8 *>(src + L::kOffsetV + (m * kPage + 16 * r + 8 * u) * 2);
                if (valid < kPage) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) off[e] = 16 * r + 8 * u + e < valid ? off[e] : (_Float16)0.0f;
                }
            } else if (m == 15) {
#pragma unroll
                for (int e = 0; e < 8; ++e) off[e] = (_Float16)1.0f;
            }
            rest = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, pv[u], rest, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const u32x4 c = *reinterpret_cast<const u32x4 *>(src + L::kCodesV + (j * 64 + lane) * 16);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                h8 p;
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = (_Float16)(sc[8 * u + e] * (float)step[j][u][e]);
                const uint32_t c0 = c[2 * u], c1 = c[2 * u + 1];
                const u32x4 lo = {c0 & mask_lo, (c0 >> 8) & mask_lo, c1 & mask_lo, (c1 >> 8) & mask_lo};
                const u32x4 hi = {c0 & mask_hi, (c0 >> 8) & mask_hi, c1 & mask_hi, (c1 >> 8) & mask_hi};
                acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, lo), p, acc[2 * j], 0, 0, 0);
                acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, hi), p, acc[2 * j + 1], 0, 0, 0);
                eights[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight, p, eights[j], 0, 0, 0);
            }
        }
        wait_copies<63>();
        if (i + R::DEPTH < count) copy(i + R::DEPTH, slot, 1);
    }

    // ---- the four wavefronts meet in LDS: [wave][m][PITCH] = output row m (2^14 times, unnormalized), then (maximum, sum)
    __syncthreads();  // (all are done with their rings)
    float *mine = lds + ((size_t)wave * 16 + m) * PITCH;
    const float back = 16777216.0f / lower;
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const float off = __shfl(rest[j & 3], (j >> 2) * 16 + m, 64);
        v4f lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = fmaf(acc[2 * j][i] - eights[j][i], back, off);
            hi[i] = fmaf(acc[2 * j + 1][i] * 0.0625f - eights[j][i], back, off);
        }
        *reinterpret_cast<v4f *>(mine + 32 * j + 4 * r) = lo;
        *reinterpret_cast<v4f *>(mine + 32 * j + 16 + 4 * r) = hi;
    }
    if (r == 3) {
        mine[D] = run_max;
        mine[D + 1] = rest[3];
    }
    __syncthreads();
    const int rows = min(16, blk.rows - row0), chunks = max(1, (blk.pages + a.chunk_pages - 1) / a.chunk_pages);
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int mm = e / (D / 4), dd = 4 * (e % (D / 4));
        const float *row = lds + (size_t)mm * PITCH;
        float f[4], mx = kNothingYet, l = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            f[x] = row[(size_t)x * 16 * PITCH + D];
            mx = fmaxf(mx, f[x]);
        }
        v4f o = {};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const v4f part = *reinterpret_cast<const v4f *>(row + (size_t)x * 16 * PITCH + dd);
            f[x] = __builtin_amdgcn_exp2f(f[x] - mx);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += f[x] * part[i];
            l += f[x] * row[(size_t)x * 16 * PITCH + D + 1];
        }
        if (chunks == 1) {
            const int s = (row0 + mm) / a.g, j = (row0 + mm) % a.g;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;  // (a row that sees nothing: 0)
            *reinterpret_cast<h4 *>(a.out + ((size_t)(blk.span.first + s) * a.h_q + kv * a.g + j) * D + dd) =
                h4{(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
        } else {
            const size_t p = ((size_t)group * a.chunks + chunk) * a.max_rows + row0 + mm;
            *reinterpret_cast<v4f *>(a.ws_o + p * D + dd) = o;
            if (dd == 0) {
                a.ws_ml[p * 2] = mx;
                a.ws_ml[p * 2 + 1] = l;
            }
        }
    }
}

// One wavefront per query row and 64 columns: lane c takes the (maximum, sum) of chunk c (at most 64).
template <int D>
__global__ __launch_bounds__(64) void attn_q4_combine_kernel(AttnQ4Args a) {
    const int lane = threadIdx.x, row = blockIdx.x, group = blockIdx.y;
    const int b = group / a.h_kv, kv = group % a.h_kv;
    const RowBlock blk = row_block(a, b, row & ~15);
    const int chunks = (blk.pages + a.chunk_pages - 1) / a.chunk_pages;
    if (row >= blk.rows || chunks <= 1) return;  // (one chunk: written by the first kernel)
    const size_t slot = (size_t)group * a.chunks * a.max_rows + row;
    const int col = 64 * blockIdx.z + lane;
    float mx = kNothingYet, l = 0.0f;
    if (lane < chunks) {
        mx = a.ws_ml[(slot + (size_t)lane * a.max_rows) * 2];
        l = a.ws_ml[(slot + (size_t)lane * a.max_rows) * 2 + 1];
    }
    float top = mx;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float f = lane < chunks ? __builtin_amdgcn_exp2f(mx - top) : 0.0f;
    float sum = f * l;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    float o = 0.0f;
    for (int c = 0; c < chunks; ++c) o = fmaf(__shfl(f, c, 64), a.ws_o[(slot + (size_t)c * a.max_rows) * D + col], o);
    const int s = row / a.g, j = row % a.g;
    a.out[((size_t)(blk.span.first + s) * a.h_q + kv * a.g + j) * D + col] = (_Float16)(sum > 0.0f ? o / sum : 0.0f);
}

template <int D>
hipError_t launch(const AttnQ4Args &a, hipStream_t st) {
    constexpr size_t lds = Ring<D>::LDS;
    if (const hipError_t e = allow_dynamic_lds<attn_q4_kernel<D>>(lds); e != hipSuccess) return e;
    attn_q4_kernel<D><<<(unsigned)((long)a.chunks * a.req.batch * a.h_kv * a.blocks), 256, lds, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.chunks == 1) return e;
    attn_q4_combine_kernel<D><<<dim3((unsigned)a.max_rows, (unsigned)(a.req.batch * a.h_kv), D / 64), 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

AttnQ4Plan plan_attention_q4(int batch, int h_kv, int g, int max_tokens, int max_context, int num_cus) {
    AttnQ4Plan p;
    const int pages = (max_context + kPage - 1) / kPage;
    p.rows = max_tokens * g;
    p.blocks = (p.rows + 15) / 16;
    const long work = (long)batch * h_kv * p.blocks, want = 4L * num_cus;
    long chunks = work >= want ? 1 : want / work;
    if (const int forced = tuning().attn_q4_chunks; forced > 0) chunks = forced < pages ? forced : pages;
    else if (chunks > (pages + 3) / 4) chunks = (pages + 3) / 4;
    if (chunks > kAttnMaxSplits) chunks = kAttnMaxSplits;
    if (chunks < 1) chunks = 1;
    p.chunk_pages = (int)((pages + chunks - 1) / chunks);
    if (p.chunk_pages < 1) p.chunk_pages = 1;
    p.chunks = (pages + p.chunk_pages - 1) / p.chunk_pages;
    if (p.chunks < 1) p.chunks = 1;
    return p;
}

size_t attention_q4_workspace(const AttnQ4Plan &p, int batch, int h_kv, int d) {
    if (p.chunks == 1) return 256;
    return (size_t)batch * h_kv * p.chunks * p.rows * (d + 2) * sizeof(float);
}

hipError_t launch_attention_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const void *pages, const AttnQ4Plan &p, void *workspace, void *out,
                               hipStream_t st) {
    AttnQ4Args a;
    a.q = static_cast<const _Float16 *>(q);
    a.out = static_cast<_Float16 *>(out);
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv;
    a.chunks = p.chunks, a.chunk_pages = p.chunk_pages, a.blocks = p.blocks, a.max_rows = p.rows;
    a.ws_o = static_cast<float *>(workspace);
    a.ws_ml = a.ws_o + (size_t)req.batch * h_kv * p.chunks * p.rows * d;
    a.scale = 1.4426950408889634f / sqrtf((float)d);
    switch (d) {
        case 64: return launch<64>(a, st);
        case 128: return launch<128>(a, st);
        case 256: return launch<256>(a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace qfc
