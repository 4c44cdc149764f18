// Which pages of a paged 4-bit cache are worth attention's while: bounds of each page's keys, and the pages whose bounds promise a query the largest scores.
//
// Bounds of a page and KV head: the largest and the smallest value hi_d, lo_d of each of its d components over the page's positions, as 8-bit codes rounded outward:
//   a = max_d max(|hi_d|, |lo_d|), step = a / 127, codes ceil(hi_d (127 / a)) and floor(lo_d (127 / a)).
// No key k of the page has q . k above sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d.  With q in 8 bits too (s_h = max |q| / 127, codes rounded to the nearest) that sum is one of whole numbers
// below 2^24, two runs of v_mfma_i32_16x16x64_i8 (the positive codes against the upper bounds, the negative ones against the lower), and exact in whatever order; a page's score for a
// token and KV head is the most any of the head's queries could reach, step max_h s_h sum_h, each product rounded to 32 bits.
#include <algorithm>

#include "paged_q4.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct BoundArgs {
    const char *pages;
    Requests req;
    int8_t *codes;  // [num_pages][h_kv][2][D]: upper, lower
    float *steps;   // [num_pages][h_kv]
    int h_kv, slots;  // pages that a request's new tokens are in, at most
};

// largest (or smallest, of negated values) over the 16 lanes of a row
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xF, 0xF, false)));  // row_ror 8, 4, 2, 1
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xF, 0xF, false)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xF, 0xF, false)));
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xF, 0xF, false)));
}
__device__ __forceinline__ int clamped(float x) { return (int)fminf(fmaxf(x, -127.0f), 127.0f); }

// A workgroup per page and head, a wavefront of it for one group of 32 values (two of eight groups).  Lane (m, r) reads what it reads in attention: of the positions of its slots the octets
// 32 j + 8 r.  Bound: latency, arrays, table, page one behind the other (one new page of each of 32 requests 6 us; a wavefront per page, with all its groups, 10).
template <int D>
__global__ __launch_bounds__(256) void bound_pages_kernel(BoundArgs a) {
    typedef PageLayout<D> L;
    constexpr int G = L::G, WAVES = G < 4 ? G : 4, J = G / WAVES;
    __shared__ float tops[2][WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, r = lane >> 4;
    const long all = (long)a.req.batch * a.slots * a.h_kv;
    int turn = 0;
    for (long i = blockIdx.x; i < all; i += gridDim.x) {
        const int kv = (int)(i % a.h_kv), slot = (int)(i / a.h_kv % a.slots), b = (int)(i / a.h_kv / a.slots);
        const Span s = span_of(a.req, b);
        const int p0 = max(s.positions - s.count, 0) / kPage + slot;
        if (s.count == 0 || p0 * (long)kPage >= s.positions) continue;
        const int page = page_of(a.req, b, p0 * kPage), there = s.positions - p0 * kPage;
        if (page < 0) continue;
        const char *src = a.pages + ((size_t)page * a.h_kv + kv) * L::kBytes;
        // (everything is asked for before any of it is looked at)
        uint32_t c[4][J];
        _Float16 by[4][J], off[4][J];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int p = 16 * (m >> 2) + 4 * t + (m & 3);
#pragma unroll
            for (int k = 0; k < J; ++k) {
                const int j = wave + WAVES * k;
                c[t][k] = *reinterpret_cast<const uint32_t *>(src + L::code_k(p, j, r));
                by[t][k] = *reinterpret_cast<const _Float16 *>(src + L::step_k(p, j));
                off[t][k] = *reinterpret_cast<const _Float16 *>(src + L::offset_k(p, j));
            }
        }
        float hi[J][8], lo[J][8], most = 0.0f;  // (lo: negated)
#pragma unroll
        for (int k = 0; k < J; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hi[k][e] = lo[k][e] = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float x = fmaf((float)((c[t][k] >> nibble(e)) & 15u) - 8.0f, (float)by[t][k], (float)off[t][k]);
                    const bool mine = 16 * (m >> 2) + 4 * t + (m & 3) < there;
                    hi[k][e] = fmaxf(hi[k][e], mine ? x : -INFINITY), lo[k][e] = fmaxf(lo[k][e], mine ? -x : -INFINITY);
                }
                hi[k][e] = row_max(hi[k][e]), lo[k][e] = row_max(lo[k][e]);
                most = fmaxf(most, fmaxf(fabsf(hi[k][e]), fabsf(lo[k][e])));
            }
        most = over_rows(most);
        turn ^= 1;  // (the next page's go beside these: one barrier is enough)
        if (lane == 0) tops[turn][wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, tops[turn][w]);
        const float f = most > 0.0f ? 127.0f / most : 0.0f;
        int8_t *dst = a.codes + ((size_t)page * a.h_kv + kv) * (2 * D);
#pragma unroll
        for (int k = 0; k < J; ++k) {  // lane m = 2 k: the upper bounds' octet, 2 k + 1: the lower ones'
            if (m >> 1 != k) continue;
            const bool upper = (m & 1) == 0;
            u32x2 codes = {0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) codes[e / 4] |= (uint32_t)(clamped(upper ? ceilf(hi[k][e] * f) : floorf(-lo[k][e] * f)) & 255) << (8 * (e % 4));
            *reinterpret_cast<u32x2 *>(dst + (upper ? 0 : D) + 32 * (wave + WAVES * k) + 8 * r) = codes;
        }
        if (threadIdx.x == 0) a.steps[(size_t)page * a.h_kv + kv] = most / 127.0f;
    }
}

struct SelectArgs {
    const _Float16 *q;
    Requests req;
    const int8_t *codes;
    const float *steps;
    int *selected;  // [tokens][h_kv][count]
    float *scores;  // [items of a slice][most_pages], where scores and list are launches of their own
    int h_q, h_kv, g, first, last, count, most_pages;
    long item0, items;  // tokens and heads of this launch
    int pieces;         // workgroups of an item's scores
};

__device__ __forceinline__ uint32_t key_of(float x) {  // order of floats as one of whole numbers
    const uint32_t u = __float_as_uint(x);
    return u ^ ((int)u < 0 ? 0xFFFFFFFFu : 0x80000000u);
}

// Largest over the wavefront
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false));  // row_ror 8, 4, 2, 1
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xF, 0xF, false));
    const u32x2 y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(y.x, y.y);
    const u32x2 z = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane(max(z.x, z.y));
}
__device__ __forceinline__ int lower(uint64_t bits) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0)); }

// The k largest of scores mid0 .. mid1 - 1 (64 R at most, more than k), of equal ones the first, ascending: by one wavefront, 64 at a time in its registers.  The range of the keys is cut into 64
// bins, the bin of the k-th into 64 again and so on; as soon as a bin ends with the k-th, those down to it are the ones (mostly after two rounds.  500 scores: 1 us; by halving 3 us, and a byte
// at a time by 16 wavefronts, with three barriers and many atomics on few words each, 5 us).
template <int R>
__device__ __forceinline__ void pick(const float *scores, int mid0, int mid1, int k, int lane, int *bins, int *out) {
    uint32_t key[R], least = 0, most = 0;  // (least: complemented)
#pragma unroll
    for (int i = 0; i < R; ++i) {
        key[i] = key_of(scores[min(mid0 + 64 * i + lane, mid1 - 1)]);  // (the last again, for the lanes behind it: loads without branches between them)
        least = max(least, ~key[i]), most = max(most, key[i]);
    }
    uint32_t lo = ~wave_max(least);
    uint32_t range = wave_max(most) - lo;  // keys lo .. lo + range are in the bins, those above them are counted
    int shift = range >= 64 ? 26 - __builtin_clz(range) : 0, above = 0, left = 0;  // (range >> shift is below 64)
    for (;;) {
        bins[lane] = 0;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint32_t over = key[i] - lo;
            if (mid0 + 64 * i + lane < mid1 && key[i] >= lo && over <= range) atomicAdd(bins + (63 - (over >> shift)), 1);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        const int own = __hip_atomic_load(bins + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT), upto = above + sum_upto(own);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
        const int l = (int)__ffsll((unsigned long long)__ballot(upto >= k)) - 1;  // (the bins hold the k-th)
        lo += (uint32_t)(63 - l) << shift;
        const int to = __builtin_amdgcn_readlane(upto, l);
        if (to == k) {
            lo -= 1;  // (all above this)
            break;
        }
        above = to - __builtin_amdgcn_readlane(own, l);
        if (shift == 0) {
            left = k - above;  // lo is the k-th: of those level with it
            break;
        }
        range = (1u << shift) - 1;
        shift = max(shift - 6, 0);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int p = mid0 + 64 * i + lane;
        const bool is_above = p < mid1 && key[i] > lo;
        const uint64_t above_bits = __ballot(is_above);
        if (left > 0) {
            const bool is_level = p < mid1 && key[i] == lo;
            const uint64_t level_bits = __ballot(is_level);
            const int level_before = lower(level_bits), of_level = min((int)__popcll(level_bits), left);
            if (is_above || (is_level && level_before < left)) out[lower(above_bits) + min(level_before, left)] = p;
            out += (int)__popcll(above_bits) + of_level;
            left -= of_level;
        } else {
            if (is_above) out[lower(above_bits)] = p;
            out += (int)__popcll(above_bits);
        }
    }
}
constexpr int kPicked = 512;  // scores that one wavefront picks from

// The same by the wavefronts of a workgroup, each with a run of the scores (from .. to - 1 of mid0 .. mid1 - 1, in order), which it reads again in every round: at(p).  bins: 4 sets of 64, zeros;
// places: two words per wavefront.  A round has one barrier: its bins are another set's than those that are read, and those that were read are zeroed.  (8 lists of 8000 scores, with the launch
// that makes these, 20 us; a byte at a time, four rounds of three barriers and all scores counted at few words, 39.  2000 scores 1.4 us less than by one wavefront from 32 registers.)
template <class At>
__device__ __forceinline__ void pick_together(const At &at, int from, int to, int k, int lane, int wave, int waves, int *bins, int (*places)[2], int *out) {
    uint32_t least = 0, most = 0;  // (least: complemented)
#pragma unroll 4
    for (int p = from + lane; p < to; p += 64) {
        const uint32_t key = key_of(at(p));
        least = max(least, ~key), most = max(most, key);
    }
    least = wave_max(least), most = wave_max(most);
    if (lane == 0) places[wave][0] = (int)least, places[wave][1] = (int)most;
    __syncthreads();
    for (int w = 0; w < waves; ++w) least = max(least, (uint32_t)places[w][0]), most = max(most, (uint32_t)places[w][1]);
    uint32_t lo = __builtin_amdgcn_readfirstlane(~least);
    uint32_t range = __builtin_amdgcn_readfirstlane(most) - lo;
    int shift = range >= 64 ? 26 - __builtin_clz(range) : 0, above = 0, left = 0;  // (range >> shift is below 64)
    for (int set = 0;; set = (set + 1) & 3) {
        int *const here = bins + 64 * set;
#pragma unroll 4
        for (int p = from + lane; p < to; p += 64) {
            const uint32_t key = key_of(at(p)), over = key - lo;
            if (key >= lo && over <= range) atomicAdd(here + (63 - (over >> shift)), 1);
        }
        __syncthreads();
        const int own = here[lane], upto = above + sum_upto(own);
        if (wave == 0) bins[64 * ((set + 3) & 3) + lane] = 0;  // (read in front of the barrier, used again behind two others)
        const int l = (int)__ffsll((unsigned long long)__ballot(upto >= k)) - 1;  // (the bins hold the k-th)
        lo += (uint32_t)(63 - l) << shift;
        const int upto_l = __builtin_amdgcn_readlane(upto, l);
        if (upto_l == k) {
            lo -= 1;  // (all above this)
            break;
        }
        above = upto_l - __builtin_amdgcn_readlane(own, l);
        if (shift == 0) {
            left = k - above;  // lo is the k-th: of those level with it
            break;
        }
        range = (1u << shift) - 1;
        shift = max(shift - 6, 0);
    }
    int mine = 0, level = 0;
#pragma unroll 4
    for (int p = from + lane; p < to; p += 64) {
        const uint32_t key = key_of(at(p));
        mine += key > lo, level += key == lo;
    }
    mine = __builtin_amdgcn_readlane(sum_upto(mine), 63), level = __builtin_amdgcn_readlane(sum_upto(level), 63);
    if (lane == 0) places[wave][0] = mine, places[wave][1] = level;
    __syncthreads();
    int level_before = 0;
    for (int w = 0; w < wave; ++w) out += places[w][0], level_before += places[w][1];
    out += min(level_before, left), left = max(left - level_before, 0);
    for (int p0 = from; p0 < to; p0 += 64) {
        const int p = p0 + lane;
        const uint32_t key = p < to ? key_of(at(p)) : 0;
        const bool is_above = p < to && key > lo, is_level = p < to && key == lo;
        const uint64_t above_bits = __ballot(is_above), level_bits = __ballot(is_level);
        const int of_level = min((int)__popcll(level_bits), left), level_in_front = lower(level_bits);
        if (is_above || (is_level && level_in_front < left)) out[lower(above_bits) + min(level_in_front, left)] = p;
        out += (int)__popcll(above_bits) + of_level;
        left -= of_level;
    }
}

// Scores of all pages that a token sees, and the list of those to be taken in ascending order: a workgroup per token and KV head does all of it (kAll), or several of them the scores (kScores),
// and one the rest (kList).  Bound: latency, of the requests' arrays, the table, the bounds one behind the other, and of the search's barriers.
enum { kAll, kScores, kList };
template <int D, int PHASE, bool IN_LDS>
__global__ __launch_bounds__(512) void select_pages_kernel(SelectArgs a) {
    constexpr int C = D / 64, AHEAD = 2;  // chunks of 64 components; groups of 16 pages on their way
    extern __shared__ float lds_scores[];
    __shared__ int counts[256], taken[8][2];
    __shared__ float tops[C][16], steps_of[16];
    __shared__ i32x4 codes[2][C][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, m = lane & 15, r = lane >> 4;
    const int pieces = PHASE == kScores ? a.pieces : 1;
    for (long work = blockIdx.x; work < a.items * pieces; work += gridDim.x) {
        const long in_slice = work / pieces, item = a.item0 + in_slice;
        float *const kept = PHASE == kAll ? nullptr : a.scores + (size_t)in_slice * a.most_pages;
        float *const scores = IN_LDS ? lds_scores : kept;
        const int kv = (int)(item % a.h_kv), token = (int)(item / a.h_kv);
        h8 asked[2] = {};
        auto ask = [&](int h0) __attribute__((always_inline)) {
            if (wave >= C) return;
            const _Float16 *q = a.q + ((size_t)token * a.h_q + kv * a.g + min(h0 + m, a.g - 1)) * D + 64 * wave + 16 * r;
            asked[0] = *reinterpret_cast<const h8 *>(q), asked[1] = *reinterpret_cast<const h8 *>(q + 8);
        };
        if constexpr (PHASE != kList) ask(0);  // (on their way before anything is known of the request)
        Span s;
        const int b = __builtin_amdgcn_readfirstlane(request_of_token(a.req, token, lane, s));
        if (b >= a.req.batch) return;
        if (token < s.first || token - s.first >= s.count) continue;
        const int pos = s.positions - s.count + token - s.first, sees = pos < 0 ? 0 : pos / kPage + 1;
        int *const out = a.selected + (size_t)item * a.count;
        if (sees <= a.count) {
            if (PHASE != kScores)
                for (int i = threadIdx.x; i < a.count; i += blockDim.x) out[i] = i < sees ? i : -1;
            continue;
        }
        const int k = a.count - a.first - a.last, mid0 = a.first, mid1 = sees - a.last;
        if (k > 0) {
            // ---- scores of the pages in between, 16 heads at a time
            if constexpr (PHASE != kList)
            for (int h0 = 0; h0 < a.g; h0 += 16) {
                // wavefront c has the queries' components 64 c .. + 63; all get their codes from LDS (each for itself, the 16 of a workgroup were 3 us at it)
                if (h0 > 0 || work != blockIdx.x) __syncthreads();  // (those before have been read)
                if (h0 > 0) ask(h0);
                float x[16], top = 0.0f;
                if (wave < C) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = (float)asked[e / 8][e % 8], top = fmaxf(top, fabsf(x[e]));
                    top = over_rows(top);
                    if (r == 0) tops[wave][m] = top;
                }
                __syncthreads();
                if (wave < C) {
#pragma unroll
                    for (int c = 0; c < C; ++c) top = fmaxf(top, tops[c][m]);
                    const float f = top > 0.0f ? 127.0f / top : 0.0f;
                    i32x4 up = {0, 0, 0, 0}, down = {0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int code = clamped(rintf(x[e] * f));
                        up[e / 4] |= (max(code, 0) & 255) << (8 * (e % 4));
                        down[e / 4] |= (min(code, 0) & 255) << (8 * (e % 4));
                    }
                    codes[0][wave][lane] = up, codes[1][wave][lane] = down;
                    if (wave == 0 && r == 0) steps_of[m] = top / 127.0f;
                }
                __syncthreads();
                i32x4 up[C], down[C];
                float of_row[4];
#pragma unroll
                for (int c = 0; c < C; ++c) up[c] = codes[0][c][lane], down[c] = codes[1][c][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) of_row[i] = steps_of[4 * r + i];
                for (int p0 = mid0 + ((int)(work % pieces) * waves + wave) * (16 * AHEAD); p0 < mid1; p0 += pieces * waves * (16 * AHEAD)) {
                    int page[AHEAD];
                    float step[AHEAD];
                    i32x4 bound[AHEAD][2 * C];
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) page[u] = page_of(a.req, b, min(p0 + 16 * u + m, mid1 - 1) * kPage);
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        const size_t at = (size_t)max(page[u], 0) * a.h_kv + kv;
#pragma unroll
                        for (int c = 0; c < 2 * C; ++c) bound[u][c] = *reinterpret_cast<const i32x4 *>(a.codes + at * (2 * D) + 64 * c + 16 * r);
                        step[u] = a.steps[at];
                    }
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) asm volatile("" : "+v"(step[u]), "+v"(bound[u][0]));  // (asked for here, not in front of their use behind each other's waits)
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        i32x4 sum = {0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[c], bound[u][c], sum, 0, 0, 0);
                            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[c], bound[u][C + c], sum, 0, 0, 0);
                        }
                        float most = (float)sum[0] * of_row[0];  // rows 4 r .. + 3, page m
#pragma unroll
                        for (int i = 1; i < 4; ++i) most = fmaxf(most, (float)sum[i] * of_row[i]);
                        most = over_rows(most);
                        most = page[u] < 0 ? -INFINITY : most * step[u];
                        const int p = p0 + 16 * u + m;
                        if (r == 0 && p < mid1) scores[p] = h0 == 0 ? most : fmaxf(scores[p], most);
                    }
                }
            }
            if constexpr (PHASE == kScores) continue;
            if (mid1 - mid0 <= kPicked) {
                __syncthreads();
                if (wave == 0) {
                    const float *from = PHASE == kList ? kept : scores;
                    const int n = mid1 - mid0;
                    if (n <= 128)
                        pick<2>(from, mid0, mid1, k, lane, counts, out + a.first);
                    else
                        pick<8>(from, mid0, mid1, k, lane, counts, out + a.first);
                }
            } else {
                const int run = ((mid1 - mid0 + waves - 1) / waves + 63) / 64 * 64, from = min(mid0 + wave * run, mid1), to = min(from + run, mid1);
                if constexpr (PHASE == kList && IN_LDS)  // (a wavefront reads what it has written)
#pragma unroll 4
                    for (int p = from + lane; p < to; p += 64) scores[p] = kept[p];
                for (int i = threadIdx.x; i < 256; i += blockDim.x) counts[i] = 0;
                __syncthreads();
                pick_together([&](int p) __attribute__((always_inline)) { return scores[p]; }, from, to, k, lane, wave, waves, counts, taken, out + a.first);
            }
        }
        if constexpr (PHASE == kScores) continue;
        for (int i = threadIdx.x; i < a.first + a.last; i += blockDim.x) out[i < a.first ? i : k + i] = i < a.first ? i : sees - (a.first + a.last) + i;
        __syncthreads();
    }
}

int pages_below(int max_context) { return (max_context + kPage - 1) / kPage; }

// Tokens and heads whose scores are kept in memory at a time
constexpr int kSlice = 512;
// One launch where scores fit the LDS and a workgroup has them at once, or workgroups are as many as half the compute units; else scores and lists are launches of their own.  One and two, us, heads
// of 128 values: 8 lists of 500 pages 10.1 and 9.1, 32 of 500 10.2 and 9.5, 128 of 500 10.7 and 11.2; 8 of 1000 15.4 and 10.2, 64 of 2000 29.1 and 19.3, 128 of 2000 29.3 and 26.4, 248 of 2000 31.6
// and 40.4.
constexpr int kOneLaunch = 512;  // pages
bool one_launch(long items, int pages, int num_cus) { return pages <= kSelectInLds && (pages <= kOneLaunch || 2 * items > num_cus); }

template <int D, int PHASE, bool IN_LDS>
hipError_t launch_phase(const SelectArgs &a, int threads, long wgs, hipStream_t st) {
    if constexpr (IN_LDS)
        if (const hipError_t e = allow_dynamic_lds<select_pages_kernel<D, PHASE, true>>((size_t)kSelectInLds * sizeof(float)); e != hipSuccess) return e;
    const long most = 1L << 20;
    select_pages_kernel<D, PHASE, IN_LDS><<<(unsigned)(wgs < most ? wgs : most), threads, IN_LDS ? (size_t)a.most_pages * sizeof(float) : 0, st>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_select(SelectArgs a, int num_cus, hipStream_t st) {
    const int threads = a.most_pages <= 128 ? 256 : 512;  // (32 pages of a wavefront are on their way at once)
    if (one_launch(a.items, a.most_pages, num_cus)) return launch_phase<D, kAll, true>(a, threads, a.items, st);
    const long all = a.items;
    for (; a.item0 < all; a.item0 += kSlice) {
        a.items = all - a.item0 < kSlice ? all - a.item0 : kSlice;
        // 128 pages are on their way to the wavefronts of a workgroup at once; four workgroups per compute unit have them (as many as there are pieces: 4 requests of 16000 pages 54 us, so 48)
        a.pieces = (int)std::min((a.most_pages + 127L) / 128, std::max(1L, (4L * num_cus + a.items - 1) / a.items));
        if (const hipError_t e = launch_phase<D, kScores, false>(a, 256, a.items * a.pieces, st); e != hipSuccess) return e;
        const hipError_t e = a.most_pages <= kSelectInLds ? launch_phase<D, kList, true>(a, 512, a.items, st) : launch_phase<D, kList, false>(a, 512, a.items, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_bound_pages_q4(const Requests &req, int h_kv, int d, const void *pages, int8_t *codes, float *steps, hipStream_t st) {
    BoundArgs a;
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.codes = codes, a.steps = steps, a.h_kv = h_kv;
    a.slots = (req.max_tokens < req.max_context ? req.max_tokens : req.max_context) / kPage + 2;
    const long wgs = (long)req.batch * a.slots * h_kv, most = 1L << 22;
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
    if (d == 64)
        bound_pages_kernel<64><<<grid, 128, 0, st>>>(a);
    else if (d == 128)
        bound_pages_kernel<128><<<grid, 256, 0, st>>>(a);
    else
        bound_pages_kernel<256><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

size_t select_workspace(int tokens, int h_kv, int max_context) {
    const int pages = pages_below(max_context);
    const long items = (long)tokens * h_kv, kept = items < kSlice ? items : kSlice;
    return 256 + (pages <= kOneLaunch ? 0 : (size_t)kept * pages * sizeof(float));  // (what any call of as many tokens and pages or fewer needs)
}

hipError_t launch_select_pages_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const int8_t *codes, const float *steps, int first, int last, int count, void *workspace,
                                  int *selected, int num_cus, hipStream_t st) {
    SelectArgs a = {};
    a.q = static_cast<const _Float16 *>(q);
    a.req = req;
    a.codes = codes, a.steps = steps, a.selected = selected, a.scores = static_cast<float *>(workspace);
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv, a.first = first, a.last = last, a.count = count, a.most_pages = pages_below(req.max_context);
    a.items = (long)req.tokens * h_kv;
    switch (d) {
        case 64: return launch_select<64>(a, num_cus, st);
        case 128: return launch_select<128>(a, num_cus, st);
        case 256: return launch_select<256>(a, num_cus, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace qfc
