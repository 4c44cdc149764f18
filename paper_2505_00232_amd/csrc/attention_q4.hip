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

constexpr int kWhole = 4;  // pages of a unit that is not cut, of small shares (256 requests of up to 150 positions 17 us, cut 33)

struct AttnQ4Args {
    const _Float16 *q;  // [tokens, h_q, D]
    _Float16 *out;
    const char *pages;
    Requests req;
    float *ws_o, *ws_ml;  // [workers, 2, 16, D] partial outputs, [.., 2] (maximum, sum)
    int h_q, h_kv, g, workers, least, whole;
    int most;  // places that requests within the call's limits have at most
    float scale;
};

// Sums of places end at the largest int.  Requests whose arrays overlap may have more places than a call's limits allow: what lies behind those (AttnQ4Args::most, 2^24 and more below
// the largest int, so that no place of a unit that is worked on passes it) is left out.
__device__ __forceinline__ int add(int x, int y) { return __builtin_elementwise_add_sat(x, y); }
// sum over the lanes up to this one
__device__ __forceinline__ int sum_upto(int x) {
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));  // row_shr 1, 2, 4, 8
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));  // row_bcast 15, 31
    x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
    return x;
}
// The work: units of a KV head and a block of 16 query rows of a request, one behind the other, each with the pages that its last row sees.  A request's blocks come in pairs, the
// first with the last and so on, all heads of a pair in turn: every pair of a request has about as many pages, so that a place in the run of all is found without a list.
// The pages are dealt to the wavefronts in equal shares (at least `least`), whatever the requests' lengths: each has one run of pages, across units.  A
// unit is done by one wavefront where it is short (half a share, or, of small shares, kWhole pages: less work than a second launch), by that in whose share it begins; of a longer
// one a wavefront does the pages of its share, and leaves partial results where others have the rest: two per wavefront at most, of the unit that its share begins inside of (or
// with), and of the one that it ends inside of.  A unit's beginning costs about as much as two pages (its requests' arrays, queries and first page one after the other): where a share
// is some pages, units are that much longer (32 requests of up to 8192 positions 46.8 us, without 49.6).
struct Unit {
    int b, kv, row0;  // b < 0: behind the last
    int begin, end;   // places in the run of all units; a unit without rows: places that are nobody's
    Span span;
};
struct Units {
    const AttnQ4Args a;
    const int lane;
    int share, over;           // pages of a wavefront, and what a unit has on top of its own
    int b0, before, before_u;  // 64 requests at a time: the first, and places and units before them
    int blocks, pages, upto, upto_u;  // of this lane's request: blocks of 16 rows, pages of a pair (of the block, where it is the only one); places and units up to its end
    Span span;
    __device__ __forceinline__ Units(const AttnQ4Args &args, int l) : a(args), lane(l), share(0), over(0), b0(0), before(0), before_u(0) {
        int all = 0, units = 0;
        for (int c = 0; c < a.req.batch; c += 64) {
            load(c);
            all = add(all, pairs(blocks) * a.h_kv * pages);
            units = add(units, pairs(blocks) * a.h_kv * of_pair(blocks));
        }
        all = last(sum_upto(all)), units = min(last(sum_upto(units)), INT32_MAX / 2);
        over = all / 4 >= a.workers ? 2 : 0;
        share = max(a.least, (min(add(all, over * units), a.most) + a.workers - 1) / a.workers);
        if (a.req.batch > 64) load(0);
        sum();
    }
    __device__ static __forceinline__ int last(int x) { return __builtin_amdgcn_readlane(x, 63); }
    __device__ static __forceinline__ int pairs(int blocks) { return (blocks + 1) / 2; }
    __device__ static __forceinline__ int of_pair(int blocks) { return blocks > 1 ? 2 : 1; }
    // pages that the last row of block k sees (one at least: a unit without positions has its rows written)
    __device__ __forceinline__ int pages_of(const Span &s, int k) const {
        return max(1, (s.positions - s.count + min(16 * k + 15, s.count * a.g - 1) / a.g + kPage) / kPage);
    }
    __device__ __forceinline__ void load(int c) {
        b0 = c;
        blocks = 0, pages = 1, span = Span{0, 0, 0};
        const int b = c + lane;
        if (b < a.req.batch) {
            span = span_of(a.req, b);
            blocks = (span.count * a.g + 15) / 16;
            pages = max(1, (span.positions + kPage - 1) / kPage);
            if (blocks > 1) {  // (of a block k and the one as far from the end, whatever k: their last tokens add up to (16 blocks + 14) / g at most)
                const int past = span.positions - span.count;
                pages += pages_of(span, (blocks - 1) / 2);
                if (past >= 0) pages = min(pages, (2 * past + (16 * blocks + 14) / a.g) / kPage + 2);
            }
        }
    }
    __device__ __forceinline__ void sum() {
        upto = sum_upto(pairs(blocks) * a.h_kv * (pages + over * of_pair(blocks)));
        upto_u = sum_upto(pairs(blocks) * a.h_kv * of_pair(blocks));
    }
    // The unit of place x or, by_index, the x-th; x does not descend from call to call
    template <bool BY_INDEX>
    __device__ __forceinline__ Unit at(int x) {
        Unit u = {-1, 0, 0, 0, 0, {0, 0, 0}};
        auto plus = [](int p, int q) __attribute__((always_inline)) { return BY_INDEX ? add(p, q) : p + q; };  // (by place: at most x and a unit's length)
        for (;;) {
            const int of = BY_INDEX ? upto_u : upto, base = BY_INDEX ? before_u : before;
            const uint64_t past = __ballot(of > x - base);
            if (past) {
                const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
                const int n = __builtin_amdgcn_readlane(blocks, l), units = of_pair(n), len = __builtin_amdgcn_readlane(pages, l) + over * units;
                const int first = plus(before, __builtin_amdgcn_readlane(upto, l) - pairs(n) * a.h_kv * len);
                const int nth = x - (before_u + __builtin_amdgcn_readlane(upto_u, l) - pairs(n) * a.h_kv * units);
                u.span = Span{__builtin_amdgcn_readlane(span.first, l), __builtin_amdgcn_readlane(span.count, l), __builtin_amdgcn_readlane(span.positions, l)};
                // (the same in every lane: said explicitly, it stays in scalar registers)
                const int pair = __builtin_amdgcn_readfirstlane(BY_INDEX ? nth / units : (x - first) / len), k = __builtin_amdgcn_readfirstlane(pair / a.h_kv);
                const int begin = plus(first, pair * len);
                u.b = __builtin_amdgcn_readfirstlane(b0 + l);
                u.kv = __builtin_amdgcn_readfirstlane(pair - k * a.h_kv);
                u.begin = __builtin_amdgcn_readfirstlane(begin);
                u.end = __builtin_amdgcn_readfirstlane(plus(begin, len));
                if (units == 2) {  // the pair's first block, its second one (the middle block has none), places that are nobody's
                    const int cut = plus(begin, over + pages_of(u.span, k)), other = n - 1 - k, end = other > k ? plus(cut, over + pages_of(u.span, other)) : cut;
                    const int which = BY_INDEX ? (nth % 2 == 0 ? 0 : other > k ? 1 : 2) : x < cut ? 0 : x < end ? 1 : 2;
                    u.row0 = __builtin_amdgcn_readfirstlane(16 * (which == 0 ? k : which == 1 ? other : n));
                    u.begin = __builtin_amdgcn_readfirstlane(which == 0 ? begin : which == 1 ? cut : end);
                    u.end = __builtin_amdgcn_readfirstlane(which == 0 ? cut : which == 1 ? end : plus(begin, len));
                }
                return u;
            }
            if (b0 + 64 >= a.req.batch) return u;
            before = add(before, last(upto));
            before_u = add(before_u, last(upto_u));
            load(b0 + 64);
            sum();
        }
    }
    // wavefronts that have places of a unit, from the w0-th on (the last one's share ends where the call's places end)
    __device__ __forceinline__ int parts_of(const Unit &u, int w0) const { return min((u.end - 1) / share, a.workers - 1) - w0 + 1; }
    __device__ __forceinline__ bool may_cut(const Unit &u) const { return u.end - u.begin - over > max(over ? share / 2 : kWhole, a.whole); }
};
// Place of the partial results that worker w leaves of a unit
__device__ __forceinline__ size_t partial_of(const Unit &u, int w, int share) { return (size_t)w * 2 + (u.begin > w * share ? 1 : 0); }

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

// Up to 16 query rows of a KV head at a time.  The wavefronts work for themselves, each with copies of its own on the way.  Bound: memory where rows are few (32 requests of up to 8192
// positions, 32 heads on 8 of 128 values: 168 MB in 41 us, 4.1 TB/s), the some 450 vector instructions of a page and block, and little that runs beside them, where they are many
// (prompts of 1024 and 601 tokens 72 us).  Two blocks that share the codes' taking apart need more registers than two wavefronts of a SIMD have, and were slower (prompts 187 us, 167
// with one, both before blocks came in pairs).
template <int D>
__global__ __launch_bounds__(256, kWgs) void attn_q4_kernel(AttnQ4Args a) {
    typedef PageLayout<D> L;
    typedef Place<D> R;
    constexpr int G = L::G, DT = D / 16, W = L::W;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane & 15, r = lane >> 4;
    char *const keys = reinterpret_cast<char *>(lds) + wave * (2 * R::PART), *const values = keys + R::PART - R::kHalf;  // (the layout counts from the page's start)
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds + wave * (2 * R::PART));
    const int worker = (int)blockIdx.x * 4 + wave;
    if (worker >= a.workers) return;
    Units units(a, lane);
    const int from = worker * units.share, stop = from + units.share;
    for (int x = from; x < stop;) {
        const Unit unit = units.at<false>(x);
        if (__builtin_amdgcn_readfirstlane(unit.b) < 0) return;
        const bool cut = units.may_cut(unit);
        if ((!cut && unit.begin < x) || unit.row0 >= unit.span.count * a.g) {  // (another wavefront has it, or there is none)
            x = unit.end;
            continue;
        }
        const int b = __builtin_amdgcn_readfirstlane(unit.b), kv = __builtin_amdgcn_readfirstlane(unit.kv), row0 = __builtin_amdgcn_readfirstlane(unit.row0);
        const Span span = unit.span;
        const int rows = span.count * a.g, n = span.positions;
        const int sees = max(0, n - rows / a.g + min(row0 + 15, rows - 1) / a.g + 1);  // positions the unit's last row sees
        const int last = cut ? min(stop, unit.end) : unit.end;
        const bool whole = unit.begin >= from && last == unit.end;  // no other wavefront has a page of the unit
        const int page0 = max(x - unit.begin - units.over, 0), pages = min(last - unit.begin - units.over, (sees + kPage - 1) / kPage);  // the unit's pages that are taken here
        x = __builtin_amdgcn_readfirstlane(last);

        // ---- copies.  Lane i holds the number of the wavefront's i-th page (of 64 at a time)
        const int count = __builtin_amdgcn_readfirstlane(pages - page0);
        auto numbers = [&](int i) __attribute__((always_inline)) { return i + lane < count ? page_of(a.req, b, (page0 + i + lane) * kPage) : -1; };
        int ahead = numbers(0), page = __builtin_amdgcn_readlane(ahead, 0);

        // ---- queries: lane (m, r) holds q[row0 + m][32 j + 8 r .. + 7], scaled by a power of two
        const bool real = row0 + m < rows;
        const int token = real ? (row0 + m) / a.g : 0, head = kv * a.g + (real ? (row0 + m) % a.g : 0);
        const size_t at = ((size_t)(span.first + token) * a.h_q + head) * D;
        const int lim = real ? n - span.count + token + 1 : 0;  // positions the lane's row sees (none where 0 or less)
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
            const _Float16 hi = (_Float16)(s * 0.0625f), lo = (_Float16)(s * 0.0625f - (float)hi);
            sums[j] = r == 0 ? hi : r == 1 ? lo : (_Float16)0.0f;
        }

        v4f acc[DT], rest = {};
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        float run_max = kNothingYet;
        const u32x4 eight_lo = {0x80088008u, 0x80088008u, 0x80088008u, 0x80088008u}, eight_hi = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u},  // -8 as a code
                    eight_k = {0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u};
        const uint32_t mask_lo = 0x000F000Fu, mask_hi = 0x00F000F0u;

        auto copy = [&](int of, int part) __attribute__((always_inline)) {  // part 0: keys, 1: values
            const char *src = a.pages + ((size_t)max(of, 0) * a.h_kv + kv) * L::kBytes + part * R::kHalf;
#pragma unroll
            for (int c = 0; c < R::COPIES; ++c)  // (the last piece's lanes behind the part copy its end again)
                copy16_to_lds(src, (uint32_t)min(c * 1024 + lane * 16, R::kHalf - 16), lds_at + part * R::PART + c * 1024);
        };
        if (count > 0) {
            copy(page, 0);
            copy(page, 1);
        }
        for (int i = 0; i < count; ++i) {
            const int k0 = (page0 + i) * kPage;
            const bool more = i + 1 < count;
            if (more && ((i + 1) & 63) == 0) ahead = numbers(i + 1);
            const int next = __builtin_amdgcn_readlane(ahead, (i + 1) & 63);
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
                        const v4f from = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_k), qf[j], zero, 0, 0, 0);
                        h8 st[2];
                        st[0] = *reinterpret_cast<const h8 *>(keys + L::kStepK + (j * kPage + 16 * r) * 2);
                        st[1] = *reinterpret_cast<const h8 *>(keys + L::kStepK + (j * kPage + 16 * r + 8) * 2);
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t w = c[t][jw];
                            const u32x4 op = {w & mask_lo, w & mask_hi, (w >> 8) & mask_lo, (w >> 8) & mask_hi};
                            const v4f x = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, op), qf[j], from, 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 4; ++i) part[t][i] = fmaf((float)st[t >> 1][4 * (t & 1) + i], x[i], part[t][i]);
                        }
                    }
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
            bmax = fmaxf(bmax, __shfl_xor(bmax, 16, 64));
            bmax = fmaxf(bmax, __shfl_xor(bmax, 32, 64)) * to_score;  // (in units of log 2 from here on)
            auto product = [&](auto second, const float (&P)[16]) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    if constexpr (decltype(second)::value) __builtin_amdgcn_sched_barrier(0);  // (a group after the other: registers)
                    const u32x4 c = *reinterpret_cast<const u32x4 *>(values + L::kCodesV + (j * 64 + lane) * 16);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const h8 step = step_of(j, u);
                        h8 p;
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = (_Float16)fmaf(P[8 * u + e], (float)step[e], 0.0f);  // (with the sum one instruction takes 32 and 16 bits)
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
                    for (int j = 0; j < G; ++j)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            __builtin_amdgcn_sched_barrier(0);
                            const h8 step = step_of(j, u);
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
            page = next;
        }

        // ---- output row m (2^kFactor times, unnormalized), its maximum and sum
        const float back = 16777216.0f, sum = __shfl(rest[3], 48 + m, 64), inv = sum != 0.0f ? 1.0f / sum : 0.0f;  // (a row that sees nothing: 0; one of a NaN stays NaN)
        const size_t part = partial_of(unit, worker, units.share) * 16 + m;
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const float off = __shfl(rest[j & 3], (j >> 2) * 16 + m, 64);
            v4f o[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[0][i] = fmaf(acc[2 * j][i], back, off);
                o[1][i] = fmaf(acc[2 * j + 1][i], back * 0.0625f, off);
            }
            if (!real) continue;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int d = 32 * j + 16 * k + 4 * r;
                if (whole)
                    *reinterpret_cast<h4 *>(a.out + at + d) = h4{(_Float16)(o[k][0] * inv), (_Float16)(o[k][1] * inv), (_Float16)(o[k][2] * inv), (_Float16)(o[k][3] * inv)};
                else
                    *reinterpret_cast<v4f *>(a.ws_o + part * D + d) = o[k];
            }
        }
        if (real && !whole && r == 0) {
            a.ws_ml[part * 2] = run_max;
            a.ws_ml[part * 2 + 1] = sum;
        }
    }
}

// Joining costs 4 to 13 us, most of it a launch and four reads one behind the other.
// The units that several wavefronts share, a row of one (unit_rows in each) per workgroup, or one after the other.  Its four wavefronts take the
// parts in turn, lane c the (maximum, sum) of its c-th and D / 64 columns of the partial outputs; they meet in LDS.
template <int D>
__global__ __launch_bounds__(256) void attn_q4_combine_kernel(AttnQ4Args a, int unit_rows) {
    constexpr int PER = D / 64;
    typedef float cols __attribute__((ext_vector_type(PER)));
    __shared__ float outs[4][D], maxima[4], sums[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Units units(a, lane);
    for (long i = blockIdx.x;; i += gridDim.x) {
        const int in_unit = (int)(i % unit_rows);
        const Unit unit = units.at<true>((int)(i / unit_rows));
        if (unit.b < 0) return;
        const int w0 = unit.begin / units.share, parts = units.parts_of(unit, w0);
        if (w0 >= a.workers) return;  // (behind the last wavefront's places)
        if (!units.may_cut(unit) || parts <= 1) continue;  // (written by the first kernel, or without a place)
        const Span span = unit.span;
        const int row = unit.row0 + in_unit;
        if (row >= span.count * a.g) continue;
        const size_t slot0 = partial_of(unit, w0, units.share) * 16 + in_unit;  // of the first; the others begin inside the unit
        auto place = [&](int c) __attribute__((always_inline)) { return c == 0 ? slot0 : (size_t)(w0 + c) * 32 + in_unit; };
        const int own = (parts - wave + 3) / 4;  // of this wavefront: wave, wave + 4, ...
        float mx = kNothingYet, l = 0.0f;
        if (lane < own) {
            mx = a.ws_ml[place(wave + 4 * lane) * 2];
            l = a.ws_ml[place(wave + 4 * lane) * 2 + 1];
        }
        // (eight parts' columns at a time are on their way before the factors are known; parts behind the last read it again and count as nothing)
        const float *src = a.ws_o + PER * lane;
        cols part[8];
        auto fetch = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < 8; ++c) part[c] = *reinterpret_cast<const cols *>(src + place(min(wave + 4 * (c0 + c), parts - 1)) * D);
        };
        fetch(0);
        float top = mx;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float f = lane < own ? __builtin_amdgcn_exp2f(mx - top) : 0.0f;
        float sum = f * l;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        cols o = {};
        for (int c0 = 0; c0 < own; c0 += 8) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float fc = c0 + c < own ? __shfl(f, (c0 + c) & 63, 64) : 0.0f;
#pragma unroll
                for (int e = 0; e < PER; ++e) o[e] = c0 + c < own ? fmaf(fc, part[c][e], o[e]) : o[e];
            }
            if (c0 + 8 < own) fetch(c0 + 8);
        }
        __syncthreads();  // (the row before has been written)
#pragma unroll
        for (int e = 0; e < PER; ++e) outs[wave][PER * lane + e] = o[e];
        if (lane == 0) maxima[wave] = top, sums[wave] = sum;
        __syncthreads();
        if (threadIdx.x < D) {
            const float high = fmaxf(fmaxf(maxima[0], maxima[1]), fmaxf(maxima[2], maxima[3]));
            float total = 0.0f, y = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float fw = __builtin_amdgcn_exp2f(maxima[w] - high);
                total = fmaf(fw, sums[w], total);
                y = fmaf(fw, outs[w][threadIdx.x], y);
            }
            a.out[((size_t)(span.first + row / a.g) * a.h_q + unit.kv * a.g + row % a.g) * D + threadIdx.x] = (_Float16)(total != 0.0f ? y / total : 0.0f);
        }
    }
}

// The same where rows are many (a call: chunks of 40 tokens of two requests 35 us, with this kernel 40; a chunk of 300 tokens beside tokens 99 us, a workgroup per row 131): a workgroup
// per worker, for the unit that the worker's share begins inside of, if it is the first to do so; a wavefront per row.
template <int D>
__global__ __launch_bounds__(256) void attn_q4_combine_rows_kernel(AttnQ4Args a) {
    constexpr int PER = D / 64;
    typedef float cols __attribute__((ext_vector_type(PER)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Units units(a, lane);
    const int x = ((int)blockIdx.x + 1) * units.share;
    const Unit unit = units.at<false>(x);
    if (unit.b < 0 || unit.begin >= x || x - unit.begin > units.share || !units.may_cut(unit)) return;
    const Span span = unit.span;
    if (unit.row0 >= span.count * a.g) return;  // (places that are nobody's)
    const int w0 = unit.begin / units.share, parts = units.parts_of(unit, w0), rows = min(16, span.count * a.g - unit.row0);
    const size_t slot0 = partial_of(unit, w0, units.share) * 16;
    // (four rows of a wavefront; everything's first parts are on their way at once, and those behind the last are read again and count as nothing)
    auto place = [&](int row, int c) __attribute__((always_inline)) { return (c == 0 ? slot0 : (size_t)(w0 + c) * 32) + min(wave + 4 * row, rows - 1); };
    float mx[4], l[4];
    cols part[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mx[i] = a.ws_ml[place(i, min(lane, parts - 1)) * 2];
        l[i] = a.ws_ml[place(i, min(lane, parts - 1)) * 2 + 1];
#pragma unroll
        for (int c = 0; c < 2; ++c) part[i][c] = *reinterpret_cast<const cols *>(a.ws_o + place(i, c) * D + PER * lane);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float top = mx[i];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float f = lane < parts ? __builtin_amdgcn_exp2f(mx[i] - top) : 0.0f;
        float sum = f * l[i];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        cols o = {};
        for (int c0 = 0; c0 < parts; c0 += 2) {
            const cols now[2] = {part[i][0], part[i][1]};
            if (c0 + 2 < parts) {
#pragma unroll
                for (int c = 0; c < 2; ++c) part[i][c] = *reinterpret_cast<const cols *>(a.ws_o + place(i, min(c0 + 2 + c, parts - 1)) * D + PER * lane);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float fc = __shfl(f, (c0 + c) & 63, 64);
#pragma unroll
                for (int e = 0; e < PER; ++e) o[e] = c0 + c < parts ? fmaf(fc, now[c][e], o[e]) : o[e];
            }
        }
        if (wave + 4 * i >= rows) return;
        const int row = unit.row0 + wave + 4 * i;
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        _Float16 *out = a.out + ((size_t)(span.first + row / a.g) * a.h_q + unit.kv * a.g + row % a.g) * D + PER * lane;
#pragma unroll
        for (int e = 0; e < PER; ++e) out[e] = (_Float16)(o[e] * inv);
    }
}

template <int D>
hipError_t launch(const AttnQ4Args &a, const AttnQ4Plan &p, int num_cus, hipStream_t st) {
    constexpr size_t lds = Place<D>::LDS;
    if (const hipError_t e = allow_dynamic_lds<attn_q4_kernel<D>>(lds); e != hipSuccess) return e;
    attn_q4_kernel<D><<<(unsigned)((a.workers + 3) / 4), 256, lds, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || !p.shared) return e;
    if (p.many) {
        if (a.workers > 1) attn_q4_combine_rows_kernel<D><<<(unsigned)(a.workers - 1), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    const int unit_rows = p.rows < 16 ? p.rows : 16;
    const long works = p.blocks * a.h_kv * unit_rows, most = 4L * num_cus;
    attn_q4_combine_kernel<D><<<(unsigned)(works < most ? works : most), 256, 0, st>>>(a, unit_rows);
    return hipGetLastError();
}

}  // namespace

AttnQ4Plan plan_attention_q4(int batch, int tokens, int h_kv, int g, int d, int max_tokens, int max_context, int num_cus) {
    AttnQ4Plan p = {};
    p.pages = (max_context + kPage - 1) / kPage;
    p.rows = max_tokens * g;
    p.blocks = p.rows <= 16 ? batch : ((long)tokens * g + 15) / 16 + 2L * batch;  // (pairs: one more where a request's number is odd)
    // as many wavefronts as the card holds at once
    const long waves = 4L * num_cus * kWgs, most_pages = p.blocks * h_kv * p.pages;
    p.many = p.blocks * h_kv * (p.rows < 16 ? p.rows : 16) > 16L * num_cus;
    const int most_shares = p.many ? 62 : 254;  // (and two ends: a lane of the combination's wavefront, or of its four, for each)
    p.least = (p.pages + most_shares) / most_shares;
    if (const int forced = tuning().attn_q4_pages; forced > p.least) p.least = forced < 1 << 20 ? forced : 1 << 20;
    const long shares = (most_pages + p.least - 1) / p.least;
    p.workers = (int)(shares < waves ? shares : waves);
    if (p.workers < 1) p.workers = 1;
    p.shared = p.pages > kWhole;
    p.bytes = 256 + (p.shared ? (size_t)p.workers * 2 * 16 * (d + 2) * sizeof(float) : 0);
    return p;
}

long most_places(const AttnQ4Plan &p, int h_kv) { return p.blocks * h_kv * (p.pages + 4); }

hipError_t launch_attention_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const void *pages, const AttnQ4Plan &p, void *workspace, void *out, int num_cus,
                               hipStream_t st) {
    AttnQ4Args a = {};
    a.q = static_cast<const _Float16 *>(q);
    a.out = static_cast<_Float16 *>(out);
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv;
    a.workers = p.workers, a.least = p.least, a.most = (int)most_places(p, h_kv), a.whole = p.shared ? 0 : INT32_MAX;  // (no second launch: nothing is cut)
    a.ws_o = static_cast<float *>(workspace);
    a.ws_ml = a.ws_o + (size_t)p.workers * 2 * 16 * d;
    a.scale = 1.4426950408889634f / sqrtf((float)d);
    switch (d) {
        case 64: return launch<64>(a, p, num_cus, st);
        case 128: return launch<128>(a, p, num_cus, st);
        case 256: return launch<256>(a, p, num_cus, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace qfc
