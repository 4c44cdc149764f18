// Attention of the new tokens of a batch of requests over their paged 4-bit cache (layout: paged_q4.h).
//
// With a cached value = offset + step (code - 8), one step and offset per 32 values (group j) of a position's head:
//   q . k = sum_j step_j (q_j . code_j - 8 sum q_j) + sum_j offset_j sum q_j
// so the score product multiplies q with the codes as they are, one v_mfma_f32_16x16x32_f16 per group: a masked nibble is the denormal code * 2^-24, the nibbles in the place 16
// times as high meet queries divided by 16, and the accumulator starts at -8 sum q_j.  The steps multiply the 32-bit result; the offsets come in by one more MFMA, against the sums of
// q in two binary16 parts (2^-22).  For the second product
//   out_d = sum_p (p step_j) (code - 8) + sum_p p offset_j
// P is multiplied with the step in 32 bits and rounded to binary16 once per group; the -8 is taken off with the same rounded values (an MFMA with a
// constant into the same sums: taken off at the end, from sums of their own, it left errors of 2^-15 of 8 steps where one position has nearly all of P), so that what the rounding
// leaves is relative to a centred code, and the offsets are again one MFMA, whose last row, ones, gives the sum of P.
// Cached values are never rounded: as binary16 copies, with the kernel for prompts over a 16-bit cache (attention.hip), prompts of 1024 and 601 tokens took 48 us instead of 76, with
// twice the error (relative to the result's norm 4.0e-4 instead of 2.8e-4, where the output's own rounding is 2.1e-4).
//
// P is taken 2^14 times as large: with steps below 2 every product is below 2^15, and binary16 keeps its 11 bits down to a product of 2^-28.  The steps of 2 and more (values some 30
// apart and more) of a page are multiplied on their own, in a turn before the others' with each row's P lowered as far as that row's products need, so that what binary16 then loses is
// little against a product that is in the row's sums; all others keep their bits.  (Where every page has such steps: 32 requests of up to 8192 positions 48 -> 61 us, prompts 76 -> 124.)
#pragma once
#include <type_traits>

#include "paged_q4.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kFactor = 14.0f;  // log 2 of what P is multiplied with
constexpr float kNothingYet = -1.0e25f;  // maximum of a row that has seen no position: below every score

// Workgroups per compute unit.  More would fit the LDS with heads of 128 and 64 values and were slower: 32 requests of up to 8192 positions 47 us, with three 51; 16 requests of 3000
// to 6000, heads of 64, 19.0, with three 21.7, with four 20.4.
constexpr int kWgs = 2;

// What a wavefront has on its way: a page's keys and its values, each in a place of PART bytes of LDS of its own, which the next page's take as soon as they are read.
template <int D>
struct Place {
    static constexpr int kHalf = 40 * D;                      // bytes of a page's keys or values
    static constexpr int PART = (kHalf + 1023) / 1024 * 1024;  // copied in pieces of a KiB
    static constexpr int COPIES = PART / 1024;
    static constexpr int LDS = 4 * 2 * PART;
    static_assert(kWgs * LDS <= 160 * 1024 && COPIES <= 63, "LDS, and the 6-bit counter of outstanding copies");
};

// 16 query rows of a KV head, their sums over the pages walked so far, and the wavefront's places in LDS.  Lane (m, r) = (lane % 16, lane / 16) has row m.
//
// SPREAD: 16 / G rows (a token's few heads), each G times, once for every group of 32 values: column m = (16 / G) a + b of the products is row b with group a's queries alone.  The products of all groups
// then go into one sum, every lane multiplies with its own group's steps (a G-th of the multiplications and of the reads of steps), and the G columns of a row are added up; P times a step is
// one product per position too, and of the second product's columns those of group a are good for the values of group a.  (Chunks of 150 and 24 tokens, 2 heads of
// 256 values on each of 4, 17 pages a token: 45 us, without 53; 32 tokens, 4 heads of 128 on each of 8, 32 pages a token: 18.6 and 19.8.)
template <int D, bool SPREAD = false>
struct Rows {
    typedef PageLayout<D> L;
    typedef Place<D> R;
    static constexpr int G = L::G, DT = D / 16, W = L::W;
    static constexpr int ROWS = SPREAD ? 16 / G : 16;
    const int lane, m, r;
    char *const keys, *const values;  // (the layout counts from the page's start)
    const uint32_t lds_at;
    h8 qf[G], sums;
    float to_score, run_max;  // (the maximum in units of log 2)
    v4f acc[DT], rest;

    __device__ __forceinline__ Rows(float *lds, int wave, int l)
        : lane(l), m(l & 15), r(l >> 4), keys(reinterpret_cast<char *>(lds) + wave * (2 * R::PART)), values(keys + R::PART - R::kHalf),
          lds_at(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds + wave * (2 * R::PART))) {}

    // Its row, and its group where SPREAD
    __device__ __forceinline__ int row() const { return m % ROWS; }
    __device__ __forceinline__ int group() const { return m / ROWS; }

    // The lane's row of the queries is q (not read where it is not `real`); scale: of scores, times log2 e.  Lane (m, r) holds q[m][32 j + 8 r .. + 7], scaled by a power of two; no position has been seen
    __device__ __forceinline__ void load(const _Float16 *q, bool real, float scale) {
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const h8 zero = {};
            qf[j] = real ? *reinterpret_cast<const h8 *>(q + 32 * j + 8 * r) : zero;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)qf[j][e]));
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        // the largest to 2^13 .. 2^14: what the division by 16 below loses is 2^-24 of it and less
        const int up = top > 0.0f ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
        const float up2 = __builtin_amdgcn_ldexpf(1.0f, up);
        to_score = __builtin_amdgcn_ldexpf(scale, 24 - up);  // 2^24: the codes' denormals
        sums = h8{};
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
            const _Float16 hi = (_Float16)(s * 0.0625f), lo = (_Float16)(s * 0.0625f - (float)hi);
            sums[j] = r == 0 ? hi : r == 1 ? lo : (_Float16)0.0f;
            if constexpr (SPREAD) {
                if (j != group()) qf[j] = h8{}, sums[j] = (_Float16)0.0f;
            }
        }

        rest = v4f{};
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        run_max = kNothingYet;
    }

    __device__ __forceinline__ void step_k(int j, h8 (&st)[2]) const {
        st[0] = *reinterpret_cast<const h8 *>(keys + L::kStepK + (j * kPage + 16 * r) * 2);
        st[1] = *reinterpret_cast<const h8 *>(keys + L::kStepK + (j * kPage + 16 * r + 8) * 2);
    }
    // sum over the columns of a row, in each of them
    __device__ static __forceinline__ float over_groups(float x) {
        static_assert(G == 2 || G == 4 || G == 8, "columns 16 / G apart, 16 in a ring");
        if constexpr (G >= 8) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x122, 0xF, 0xF, true));  // row_ror 2, 4, 8
        if constexpr (G >= 4) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x124, 0xF, 0xF, true));
        return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xF, 0xF, true));
    }

    // `count` pages of KV head kv, of which row m sees the positions below `lim` and anyone those below n.  numbers(i): page i + lane of them (-1: none), `ahead` = numbers(0);
    // start_of(i): the first position of page i, asked for in order, before numbers() of a later 64.
    template <class Numbers, class Starts>
    __device__ __forceinline__ void walk(int count, int lim, int n, const char *pages, int h_kv, int kv, int ahead, const Numbers &numbers, const Starts &start_of) {
        int page = __builtin_amdgcn_readlane(ahead, 0), k0 = start_of(0);
        const u32x4 eight_lo = {0x80088008u, 0x80088008u, 0x80088008u, 0x80088008u}, eight_hi = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u},  // -8 as a code
                    eight_k = {0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u};
        const uint32_t mask_lo = 0x000F000Fu, mask_hi = 0x00F000F0u;

        auto copy = [&](int of, int part) __attribute__((always_inline)) {  // part 0: keys, 1: values
            const char *src = pages + ((size_t)max(of, 0) * h_kv + kv) * L::kBytes + part * R::kHalf;
#pragma unroll
            for (int c = 0; c < R::COPIES; ++c)  // (the last piece's lanes behind the part copy its end again)
                copy16_to_lds(src, (uint32_t)min(c * 1024 + lane * 16, R::kHalf - 16), lds_at + part * R::PART + c * 1024);
        };
        if (count > 0) {
            copy(page, 0);
            copy(page, 1);
        }
        for (int i = 0; i < count; ++i) {
            const bool more = i + 1 < count;
            if (more && ((i + 1) & 63) == 0) ahead = numbers(i + 1);
            const int next = __builtin_amdgcn_readlane(ahead, (i + 1) & 63), next_k0 = start_of(i + 1);
            wait_copies<R::COPIES>();  // the page's keys are there: behind them are its values
            const int seen = page >= 0 ? lim - k0 : 0, valid = page >= 0 ? n - k0 : 0;  // of this page, by the lane's row and by anyone
            // ---- scores; lane (m, r), element 4 t + i: position 16 r + 4 t + i, times 2^-24 and the queries' power of two
            float sc[16];
            {
                h8 off[4] = {};
                if (r < 2) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int j = 0; j < G; ++j) off[t][j] = reinterpret_cast<const _Float16 *>(keys + L::kOffsetK + (16 * t + m) * G * 2)[j];
                }
                v4f part[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const v4f zero = {};
                    part[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(off[t], sums, zero, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[t][i] *= 1.0f / 1048576.0f;
                }
                v4f all[4];
                if constexpr (SPREAD) {
                    v4f from = {};
#pragma unroll
                    for (int j = 0; j < G; ++j) from = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_k), qf[j], from, 0, 0, 0);
#pragma unroll
                    for (int t = 0; t < 4; ++t) all[t] = from;
                }
#pragma unroll
                for (int jj = 0; jj < G / W; ++jj) {
                    typedef uint32_t words __attribute__((ext_vector_type(W)));
                    words c[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) c[t] = *reinterpret_cast<const words *>(keys + L::kCodesK + ((t * (G / W) + jj) * 64 + lane) * (4 * W));
#pragma unroll
                    for (int jw = 0; jw < W; ++jw) {
                        const int j = jj * W + jw;
                        const v4f zero = {};
                        v4f from = zero;
                        if constexpr (!SPREAD) from = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_k), qf[j], zero, 0, 0, 0);
                        h8 st[2];
                        if constexpr (!SPREAD) step_k(j, st);
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t w = c[t][jw];
                            const u32x4 op = {w & mask_lo, w & mask_hi, (w >> 8) & mask_lo, (w >> 8) & mask_hi};
                            if constexpr (SPREAD) {
                                all[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, op), qf[j], all[t], 0, 0, 0);
                            } else {
                                const v4f x = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, op), qf[j], from, 0, 0, 0);
#pragma unroll
                                for (int i = 0; i < 4; ++i) part[t][i] = fmaf((float)st[t >> 1][4 * (t & 1) + i], x[i], part[t][i]);
                            }
                        }
                    }
                }
                if constexpr (SPREAD) {
                    h8 st[2];
                    step_k(group(), st);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[t][i] = over_groups(fmaf((float)st[t >> 1][4 * (t & 1) + i], all[t][i], part[t][i]));
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[e] = part[e >> 2][e & 3];
            }
            if (__any(seen < kPage)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[e] = 16 * r + e < seen ? sc[e] : -INFINITY;
            }
            float bmax = fmaxf(sc[0], sc[1]);
#pragma unroll
            for (int e = 2; e < 16; e += 2) bmax = fmaxf(fmaxf(bmax, sc[e]), sc[e + 1]);
            wait_copies<63>();  // (in front of a copy into a place all reads of it are done)
            if (more) {
                copy(next, 0);
                wait_copies<R::COPIES>();  // the values: behind them are the next page's keys
            } else {
                wait_copies<0>();
            }
            if (valid < kPage) {  // positions that nobody has may hold anything: their values' steps and offsets are taken as 0
                if (lane >= valid) {
#pragma unroll
                    for (int j = 0; j < G; ++j) {
                        *reinterpret_cast<_Float16 *>(values + L::step_v(lane, j)) = (_Float16)0.0f;
                        *reinterpret_cast<_Float16 *>(values + L::offset_v(lane, j)) = (_Float16)0.0f;
                    }
                }
            }
            auto step_of = [&](int j, int u) __attribute__((always_inline)) { return *reinterpret_cast<const h8 *>(values + L::kStepV + (j * kPage + 16 * r + 8 * u) * 2); };
            typedef uint32_t words __attribute__((ext_vector_type(G / 2)));
            words *const steps_at = reinterpret_cast<words *>(values + L::kStepV + lane * (2 * G));  // some of the page's steps; all of them in the wavefront
            const words steps = *steps_at;
            uint32_t any = steps[0];
#pragma unroll
            for (int j = 1; j < G / 2; ++j) any |= steps[j];
            const bool twice = __any((any & 0x40004000u) != 0);  // a step of 2 or more
            auto large = [&]() __attribute__((always_inline)) { return (steps >> 14 & 0x00010001u) * 0xFFFFu; };  // the bits of those
            bmax = over_rows(bmax) * to_score;  // (in units of log 2 from here on)
            auto product = [&](auto second, const float (&P)[16]) __attribute__((always_inline)) {
                h8 own[2];
                if constexpr (SPREAD) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const h8 step = step_of(group(), u);
#pragma unroll
                        for (int e = 0; e < 8; ++e) own[u][e] = (_Float16)fmaf(P[8 * u + e], (float)step[e], 0.0f);
                    }
                }
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    if constexpr (decltype(second)::value) __builtin_amdgcn_sched_barrier(0);  // (a group after the other: registers)
                    const u32x4 c = *reinterpret_cast<const u32x4 *>(values + L::kCodesV + (j * 64 + lane) * 16);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        h8 p;
                        if constexpr (SPREAD) {
                            p = own[u];
                        } else {
                            const h8 step = step_of(j, u);
#pragma unroll
                            for (int e = 0; e < 8; ++e) p[e] = (_Float16)fmaf(P[8 * u + e], (float)step[e], 0.0f);  // (with the sum one instruction takes 32 and 16 bits)
                        }
                        const uint32_t c0 = c[2 * u], c1 = c[2 * u + 1];
                        const u32x4 lo = {c0 & mask_lo, (c0 >> 8) & mask_lo, c1 & mask_lo, (c1 >> 8) & mask_lo};
                        const u32x4 hi = {c0 & mask_hi, (c0 >> 8) & mask_hi, c1 & mask_hi, (c1 >> 8) & mask_hi};
                        acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, lo), p, acc[2 * j], 0, 0, 0);
                        acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, hi), p, acc[2 * j + 1], 0, 0, 0);
                        acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_lo), p, acc[2 * j], 0, 0, 0);
                        acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_hi), p, acc[2 * j + 1], 0, 0, 0);
                    }
                }
            };
            if (__any(bmax > run_max) || twice) {
                const float new_max = fmaxf(run_max, bmax), corr = __builtin_amdgcn_exp2f(run_max - new_max);
                run_max = new_max;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc[t][i] *= corr;
                    rest[i] *= corr;
                }
                if (twice) {  // the large steps: the row's largest product to 2^14 .. 2^15 (by powers of two: exact in P and in sums of 32 bits)
                    *steps_at = steps & large();
                    float P[16], most = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) P[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], to_score, kFactor - run_max));
#pragma unroll
                    for (int j = 0; j < (SPREAD ? 1 : G); ++j)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            __builtin_amdgcn_sched_barrier(0);
                            const h8 step = step_of(SPREAD ? group() : j, u);
#pragma unroll
                            for (int e = 0; e < 8; ++e) most = fmaxf(most, P[8 * u + e] * (float)step[e]);
                        }
                    most = fmaxf(most, __shfl_xor(most, 16, 64));
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    const int down = most >= 32768.0f ? __builtin_amdgcn_frexp_expf(most) - 15 : 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) P[e] = __builtin_amdgcn_ldexpf(P[e], -down);
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_amdgcn_ldexpf(acc[t][i], -down);
                    product(std::true_type(), P);
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_amdgcn_ldexpf(acc[t][i], down);
                    *steps_at = steps & ~large();
                }
            }
            const float from_max = kFactor - run_max;
            h8 pv[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], to_score, from_max));
                pv[e >> 3][e & 7] = (_Float16)sc[e];
            }
            // ---- second product
#pragma unroll
            for (int u = 0; u < 2; ++u) {  // rows 0 .. G - 1: offsets; row 15: ones; the others are not used
                const u32x4 w = *reinterpret_cast<const u32x4 *>(values + L::kOffsetV + (min(m, G - 1) * kPage + 16 * r + 8 * u) * 2);
                const u32x4 rows = {m == 15 ? 0x3C003C00u : w.x, m == 15 ? 0x3C003C00u : w.y, m == 15 ? 0x3C003C00u : w.z, m == 15 ? 0x3C003C00u : w.w};
                rest = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, rows), pv[u], rest, 0, 0, 0);
            }
            product(std::false_type(), sc);
            wait_copies<63>();
            if (more) copy(next, 1);
            page = next, k0 = next_k0;
        }
    }

    // Columns 32 j + 16 k + 4 r .. + 3 of row m (2^kFactor times, unnormalized) to put(column, k-th of j's values); sum(): of row m
    __device__ __forceinline__ float sum() const { return __shfl(rest[3], 48 + m, 64); }
    template <class Put>
    __device__ __forceinline__ void columns(const Put &put) const {
        const float back = 16777216.0f;
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const float off = __shfl(rest[j & 3], (j >> 2) * 16 + m, 64);
            v4f o[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[0][i] = fmaf(acc[2 * j][i], back, off);
                o[1][i] = fmaf(acc[2 * j + 1][i], back * 0.0625f, off);
            }
            if (SPREAD && j != group()) continue;  // (of the row's other columns)
#pragma unroll
            for (int k = 0; k < 2; ++k) put(32 * j + 16 * k + 4 * r, o[k]);
        }
    }
};

}  // namespace
}  // namespace qfc
