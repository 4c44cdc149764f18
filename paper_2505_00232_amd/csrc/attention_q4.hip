// Attention of the new tokens of a batch of requests over their paged 4-bit cache (layout: paged_q4.h).
//
// With a cached value = offset + step (code - 8), one step and offset per 32 values (group j) of a position's head:
//   q . k = sum_j step_j (q_j . code_j - 8 sum q_j) + sum_j offset_j sum q_j
// so the score product multiplies q with the codes as they are, one v_mfma_f32_16x16x32_f16 per group: a masked nibble is the denormal code * 2^-24, the nibbles in the place 16
// times as high meet queries divided by 16, and the accumulator starts at -8 sum q_j.  The steps multiply the 32-bit result; the offsets come in by one more MFMA, against the sums of
// q in two binary16 parts (2^-22).  For the second product
//   out_d = sum_p (p step_j) (code - 8) + sum_p p offset_j
// P is multiplied with the step in 32 bits and rounded to binary16 once per group; the -8 is taken off with the same rounded values (an MFMA with a
// constant into the same sums), so that what the rounding leaves is relative to a centred code, and the offsets are again one MFMA, whose last row, ones, gives the sum of P.
//
// Few query rows of a request (up to few_rows per KV head: tokens, short chunks) go through that kernel in blocks of 16.  Many rows would take the same
// codes apart again and again: for them the pages are first turned into binary16 copies in the workspace, once, and the kernel for prompts (attention.hip) walks
// those.  Which request is which is known on the device only, where a first small kernel finds it.
// P is taken 2^14 times as large: with steps below 2 every product is below 2^15, and binary16 keeps its 11 bits down to a product of 2^-28.  A step of 2 or more (values some 30
// apart and more) lowers that factor to 2^2 from there on, for which every step (8734 at most) is small enough.
#include "paged_q4.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kFactor = 14.0f, kLower = 12.0f;  // log 2 of what P is multiplied with, of what large steps divide that by
constexpr float kNothingYet = -1.0e25f;  // maximum of a row that has seen no position: below every score

// Rows of a request per KV head that the blocks of 16 take.  Heads 32 on 8 of 128 values, us with blocks of 16 / with copies: one request at 512 positions 128 rows 15 / 23,
// 256 rows 18 / 23, 512 rows 26 / 23, at 4096 positions 256 rows 31 / 33, 512 rows 46 / 39; eight requests, which keep the card busy, at 512 positions 128 rows 40 / 31, 192 rows
// 54 / 32, at 4096 positions 72 rows 54 / 87, 128 rows 77 / 92, 192 rows 113 / 122, 256 rows 136 / 121.
int few_rows(long all_rows) { return all_rows > 1024 ? 128 : 256; }
constexpr int kMaxSlots = 256;  // requests of many rows at most, the others go through the blocks of 16

constexpr int kWhole = 4;  // pages of a unit that is not cut, of small shares

struct AttnQ4Args {
    const _Float16 *q;  // [tokens, h_q, D]
    _Float16 *out;
    const char *pages;
    Requests req;
    float *ws_o, *ws_ml;  // [workers, 2, 16, D] partial outputs, [.., 2] (maximum, sum)
    int *plan;            // ManyRows, or null
    int h_q, h_kv, g, workers, least, whole;
    float scale;
};

// The work: units of a KV head and a block of 16 query rows of a request, one behind the other (a request's blocks, in each all heads), each with the request's
// pages.  The pages are dealt to the wavefronts in equal shares (at least `least`), whatever the requests' lengths: each has one run of pages, across units.  A
// unit is done by one wavefront where it is short (half a share, or, of small shares, kWhole pages: less work than a second launch), by that in whose share it begins; of a longer one a wavefront does the pages of its share, and
// leaves partial results where others have the rest: two per wavefront at most, of the unit that its share begins inside of (or with), and of
// the one that it ends inside of.  A unit's beginning costs about as much as two pages (its requests' arrays, queries and first page one after the other): where a share
// is some pages, units are that much longer.
__device__ __forceinline__ bool has_many(const AttnQ4Args &a, int b) { return a.plan && a.plan[ManyRows::kSlots + b] >= 0; }
// sum over the lanes up to this one
__device__ __forceinline__ int sum_upto(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}
struct Unit {
    int b, kv, row0;  // b < 0: behind the last
    int begin, end;   // places in the run of all units
    Span span;
};
struct Units {
    const AttnQ4Args a;
    const int lane;
    int share, over;           // pages of a wavefront, and what a unit has on top of its own
    int b0, before, before_u;  // 64 requests at a time: the first, and places and units before them
    int count, pages, upto, upto_u;  // of this lane's request: units, pages of each; places and units up to its end
    Span span;
    __device__ __forceinline__ Units(const AttnQ4Args &args, int l) : a(args), lane(l), share(0), over(0), b0(0), before(0), before_u(0) {
        int all = 0, units = 0;
        for (int c = 0; c < a.req.batch; c += 64) {
            load(c);
            all += count * pages;
            units += count;
        }
        all = last(sum_upto(all)), units = last(sum_upto(units));
        over = all / 4 >= a.workers ? 2 : 0;
        share = max(a.least, (all + over * units + a.workers - 1) / a.workers);
        if (a.req.batch > 64) load(0);
        sum();
    }
    __device__ static __forceinline__ int last(int x) { return __builtin_amdgcn_readlane(x, 63); }
    __device__ __forceinline__ void load(int c) {
        b0 = c;
        count = 0, pages = 1, span = Span{0, 0, 0};  // (a unit without positions counts as one page: its rows are written)
        const int b = c + lane;
        if (b < a.req.batch && !has_many(a, b)) {
            span = span_of(a.req, b);
            count = (span.count * a.g + 15) / 16 * a.h_kv;
            pages = max(1, (span.positions + kPage - 1) / kPage);
        }
    }
    __device__ __forceinline__ void sum() {
        upto = sum_upto(count * (pages + over));
        upto_u = sum_upto(count);
    }
    // The unit of place x or, by_index, the x-th; x does not descend from call to call
    template <bool BY_INDEX>
    __device__ __forceinline__ Unit at(int x) {
        Unit u = {-1, 0, 0, 0, 0, {0, 0, 0}};
        for (;;) {
            const int of = BY_INDEX ? upto_u : upto, base = BY_INDEX ? before_u : before;
            const uint64_t past = __ballot(of > x - base);
            if (past) {
                const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
                const int n = __builtin_amdgcn_readlane(count, l), len = __builtin_amdgcn_readlane(pages, l) + over;
                const int first = before + __builtin_amdgcn_readlane(upto, l) - n * len;
                const int index = BY_INDEX ? x - (before_u + __builtin_amdgcn_readlane(upto_u, l) - n) : (x - first) / len;
                // (the same in every lane: said explicitly, it stays in scalar registers)
                u.b = __builtin_amdgcn_readfirstlane(b0 + l);
                u.kv = __builtin_amdgcn_readfirstlane(index % a.h_kv);
                u.row0 = __builtin_amdgcn_readfirstlane(index / a.h_kv * 16);
                u.begin = __builtin_amdgcn_readfirstlane(first + index * len);
                u.end = __builtin_amdgcn_readfirstlane(u.begin + len);
                u.span = Span{__builtin_amdgcn_readlane(span.first, l), __builtin_amdgcn_readlane(span.count, l), __builtin_amdgcn_readlane(span.positions, l)};
                return u;
            }
            if (b0 + 64 >= a.req.batch) return u;
            before += last(upto);
            before_u += last(upto_u);
            load(b0 + 64);
            sum();
        }
    }
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

// Up to 16 query rows of a KV head at a time.  The wavefronts work for themselves, each with copies of its own on the way.
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
        if (!cut && unit.begin < x) {  // (another wavefront has it)
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
        float run_max = kNothingYet, factor = kFactor;
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
            uint32_t large;  // some of the page's steps; all of them in the wavefront
            {
                typedef uint32_t words __attribute__((ext_vector_type(G / 2)));
                const words w = *reinterpret_cast<const words *>(values + L::kStepV + lane * (2 * G));
                large = w[0];
#pragma unroll
                for (int j = 1; j < G / 2; ++j) large |= w[j];
            }
            bmax = fmaxf(bmax, __shfl_xor(bmax, 16, 64));
            bmax = fmaxf(bmax, __shfl_xor(bmax, 32, 64)) * to_score;  // (in units of log 2 from here on)
            const bool lowers = factor == kFactor && __any((large & 0x40004000u) != 0);  // a step of 2 or more
            if (__any(bmax > run_max) || lowers) {
                const float new_max = fmaxf(run_max, bmax), corr = __builtin_amdgcn_exp2f(run_max - new_max - (lowers ? kLower : 0.0f));
                run_max = new_max;
                factor = lowers ? kFactor - kLower : factor;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc[t][i] *= corr;
                    rest[i] *= corr;
                }
            }
            const float from_max = factor - run_max;
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
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const u32x4 c = *reinterpret_cast<const u32x4 *>(values + L::kCodesV + (j * 64 + lane) * 16);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const h8 step = step_of(j, u);
                    h8 p;
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = (_Float16)fmaf(sc[8 * u + e], (float)step[e], 0.0f);  // (with the sum one instruction takes 32 and 16 bits)
                    const uint32_t c0 = c[2 * u], c1 = c[2 * u + 1];
                    const u32x4 lo = {c0 & mask_lo, (c0 >> 8) & mask_lo, c1 & mask_lo, (c1 >> 8) & mask_lo};
                    const u32x4 hi = {c0 & mask_hi, (c0 >> 8) & mask_hi, c1 & mask_hi, (c1 >> 8) & mask_hi};
                    acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, lo), p, acc[2 * j], 0, 0, 0);
                    acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, hi), p, acc[2 * j + 1], 0, 0, 0);
                    acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_lo), p, acc[2 * j], 0, 0, 0);
                    acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, eight_hi), p, acc[2 * j + 1], 0, 0, 0);
                }
            }
            wait_copies<63>();
            if (more) copy(next, 1);
            page = next;
        }

        // ---- output row m (2^kFactor times, unnormalized), its maximum and sum
        const float back = 16777216.0f, sum = __shfl(rest[3], 48 + m, 64), inv = sum > 0.0f ? 1.0f / sum : 0.0f;  // (a row that sees nothing: 0)
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
        if (!units.may_cut(unit)) continue;
        const int w0 = unit.begin / units.share, parts = (unit.end - 1) / units.share - w0 + 1;
        if (parts == 1) continue;  // (written by the first kernel)
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
            a.out[((size_t)(span.first + row / a.g) * a.h_q + unit.kv * a.g + row % a.g) * D + threadIdx.x] = (_Float16)(total > 0.0f ? y / total : 0.0f);
        }
    }
}

// ---------------------------------------------------------------- many query rows
struct ManyArgs {
    Requests req;
    int *plan;
    const char *pages;
    _Float16 *kc, *vc;  // [slots, h_kv, positions, D], [slots, h_kv, positions / 64, D, 64]
    int g, h_kv, slots, records, block_rows, chunk_steps, max_pages, few;
};

// One workgroup: the list of the requests with more than `few` rows, and how many workgroups each takes (per block of rows one for a chunk of its steps).  A request with a missing
// page, or with fewer positions than tokens, is none of them: the kernel for few rows takes it.
__global__ __launch_bounds__(256) void attn_q4_list_kernel(ManyArgs a) {
    __shared__ uint64_t wanted[4];
    __shared__ int rec[kMaxSlots][4], item[kMaxSlots];
    const int tid = threadIdx.x;
    int count = 0;  // (the same in every thread)
    for (int b0 = 0; b0 < a.req.batch; b0 += 256) {
        const int b = b0 + tid;
        bool many = false;
        if (b < a.req.batch) {
            const Span s = span_of(a.req, b);
            many = s.count * a.g > a.few && s.positions >= s.count;
            if (!many) a.plan[ManyRows::kSlots + b] = -1;
        }
        const uint64_t mask = __ballot(many);
        if ((tid & 63) == 0) wanted[tid >> 6] = mask;
        __syncthreads();
        for (int w = 0; w < 4; ++w) {
            for (uint64_t m = wanted[w]; m; m &= m - 1) {
                const int bb = b0 + 64 * w + __ffsll((unsigned long long)m) - 1;
                const Span s = span_of(a.req, bb);
                bool missing = false;
                for (int p = tid; p * kPage < s.positions; p += 256) missing = missing || page_of(a.req, bb, p * kPage) < 0;
                const bool taken = !__syncthreads_or(missing) && count < a.slots;
                if (tid == 0) {
                    if (taken) rec[count][0] = s.first, rec[count][1] = s.count, rec[count][2] = s.positions, rec[count][3] = bb;
                    a.plan[ManyRows::kSlots + bb] = taken ? count : -1;
                }
                count += taken;
            }
        }
        __syncthreads();
    }
    // steps of the last row of block j of a request's rows
    auto steps = [&](int slot, int j) {
        const int S = rec[slot][1], last = min((j + 1) * a.block_rows, S * a.g) - 1;
        return (rec[slot][2] - S + last / a.g + 1 + 31) / 32;
    };
    if (tid < count) {
        const int blocks = (rec[tid][1] * a.g + a.block_rows - 1) / a.block_rows;
        int n = blocks;
        if (a.chunk_steps > 0) {
            n = 0;
            for (int j = 0; j < blocks; ++j) n += (steps(tid, j) + a.chunk_steps - 1) / a.chunk_steps;
        }
        item[tid] = n;
    }
    __syncthreads();
    if (tid == 0) {
        int sum = 0;
        for (int i = 0; i < count; ++i) {
            const int n = item[i];
            item[i] = sum;
            sum += n;
        }
        a.plan[ManyRows::kCount] = count;
        a.plan[ManyRows::kItems] = sum;
    }
    __syncthreads();
    if (tid < count) {
        int *r = a.plan + a.records + tid * ManyRows::kRecord;
        r[ManyRows::kRow] = rec[tid][0];
        r[ManyRows::kTokens] = rec[tid][1];
        r[ManyRows::kPositions] = rec[tid][2];
        r[ManyRows::kItem] = item[tid];
        r[ManyRows::kChunkSteps] = a.chunk_steps;
        r[ManyRows::kRequest] = rec[tid][3];
    }
}

// grid = (pages of the longest request x KV heads, slots): a page's block of one head as binary16, fp16(offset + step (code - 8)).  Bound: memory.
template <int D>
__global__ __launch_bounds__(256) void attn_q4_copy_kernel(ManyArgs a) {
    typedef PageLayout<D> L;
    constexpr int G = L::G;
    const int slot = blockIdx.y, kv = (int)blockIdx.x % a.h_kv, pg = (int)blockIdx.x / a.h_kv;
    if (slot >= a.plan[ManyRows::kCount]) return;
    const int *r = a.plan + a.records + slot * ManyRows::kRecord;
    if (pg * kPage >= r[ManyRows::kPositions]) return;
    const int page = page_of(a.req, r[ManyRows::kRequest], pg * kPage);
    if (page < 0) return;  // (none of the list's requests)
    const char *src = a.pages + ((size_t)page * a.h_kv + kv) * L::kBytes;
    const size_t dst = ((size_t)(slot * a.h_kv + kv) * a.max_pages + pg) * (kPage * D);
    const int tid = threadIdx.x;
    // keys: a thread per octet
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int o = (tid + 256 * i) % (D / 8), p = (tid + 256 * i) / (D / 8), j = o / 4;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(src + L::code_k(p, j, o & 3));
        const float step = (float)*reinterpret_cast<const _Float16 *>(src + L::step_k(p, j)), off = (float)*reinterpret_cast<const _Float16 *>(src + L::offset_k(p, j));
        h8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (_Float16)fmaf((float)((w >> nibble(e)) & 15u) - 8.0f, step, off);
        *reinterpret_cast<h8 *>(a.kc + dst + p * D + 8 * o) = x;
    }
    // values: a thread per 8 positions of the two values of a byte
#pragma unroll
    for (int i = 0; i < G * 128 / 256; ++i) {
        const int t = tid + 256 * i, p0 = 8 * (t % 8), m = t / 8 % 16, j = t / 128;
        const uint2 w = *reinterpret_cast<const uint2 *>(src + L::kCodesV + (j * 64 + (p0 >> 4) * 16 + m) * 16 + (p0 & 8));
        const h8 step = *reinterpret_cast<const h8 *>(src + L::step_v(p0, j)), off = *reinterpret_cast<const h8 *>(src + L::offset_v(p0, j));
        h8 lo, hi;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t byte = (e < 4 ? w.x : w.y) >> (8 * (((e & 1) << 1) | ((e >> 1) & 1)));
            lo[e] = (_Float16)fmaf((float)(byte & 15u) - 8.0f, (float)step[e], (float)off[e]);
            hi[e] = (_Float16)fmaf((float)((byte >> 4) & 15u) - 8.0f, (float)step[e], (float)off[e]);
        }
        *reinterpret_cast<h8 *>(a.vc + dst + (32 * j + m) * 64 + p0) = lo;
        *reinterpret_cast<h8 *>(a.vc + dst + (32 * j + 16 + m) * 64 + p0) = hi;
    }
}

template <int D>
hipError_t launch(const AttnQ4Args &a, const ManyArgs &many, const AttnQ4Plan &p, int num_cus, hipStream_t st) {
    if (p.slots > 0) {
        attn_q4_list_kernel<<<1, 256, 0, st>>>(many);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    constexpr size_t lds = Place<D>::LDS;
    if (const hipError_t e = allow_dynamic_lds<attn_q4_kernel<D>>(lds); e != hipSuccess) return e;
    attn_q4_kernel<D><<<(unsigned)((a.workers + 3) / 4), 256, lds, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p.shared) {
        const int unit_rows = p.rows < 16 ? p.rows : 16;
        const long works = p.blocks * a.h_kv * unit_rows, most = 4L * num_cus;
        attn_q4_combine_kernel<D><<<(unsigned)(works < most ? works : most), 256, 0, st>>>(a, unit_rows);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (p.slots > 0) {
        attn_q4_copy_kernel<D><<<dim3((unsigned)(p.pages * a.h_kv), (unsigned)p.slots), 256, 0, st>>>(many);
        return hipGetLastError();
    }
    return hipSuccess;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

AttnQ4Plan plan_attention_q4(int batch, int tokens, int h_kv, int g, int d, int max_tokens, int max_context, int num_cus) {
    AttnQ4Plan p = {};
    p.pages = (max_context + kPage - 1) / kPage;
    p.rows = max_tokens * g;
    p.all_rows = (long)tokens * g;
    p.blocks = p.rows <= 16 ? batch : (p.all_rows + 15) / 16 + batch;
    // few rows: as many wavefronts as the card holds at once
    const long waves = 4L * num_cus * kWgs, most_pages = p.blocks * h_kv * p.pages;
    p.least = (p.pages + 2 + 253) / 254;  // (a unit is cut into 254 whole shares and two ends at most: the combination's four wavefronts take 64 each)
    if (const int forced = tuning().attn_q4_pages; forced > p.least) p.least = forced;
    const long shares = (most_pages + p.least - 1) / p.least;
    p.workers = (int)(shares < waves ? shares : waves);
    if (p.workers < 1) p.workers = 1;
    p.shared = p.pages > kWhole;
    p.total = 256;
    p.partial = 0;
    if (p.shared) p.total += up256((size_t)p.workers * 2 * 16 * (d + 2) * sizeof(float));
    // many rows
    const int few = few_rows(p.all_rows);
    if (p.rows <= few) return p;
    const long most = p.all_rows / (few + 1);
    p.slots = (int)(most < batch ? most : batch);
    if (p.slots > kMaxSlots) p.slots = kMaxSlots;
    if (p.slots == 0) return p;
    // (as for equal requests of the most tokens and positions, as many as make up the rows)
    const long alike = (p.all_rows + p.rows / 2) / p.rows;
    p.shares = plan_attention_many((int)((alike < 1 ? 1 : alike) * h_kv), max_tokens, g, d, max_context, num_cus, &p.chunk_steps);
    const int steps = (max_context + 31) / 32, chunks = p.chunk_steps > 0 ? (steps + p.chunk_steps - 1) / p.chunk_steps : 1;
    p.items = (int)((p.all_rows / (128 / p.shares) + p.slots) * chunks);
    p.records = (ManyRows::kSlots + batch + 7) / 8 * 8;
    p.plan = p.total;
    p.total += up256((size_t)(p.records + p.slots * ManyRows::kRecord) * sizeof(int));
    p.copies = p.total;
    p.total += up256((size_t)p.slots * h_kv * p.pages * kPage * d * 2 * 2);
    p.many_partial = p.total;
    if (p.chunk_steps > 0) p.total += up256((size_t)kPrefillMaxChunks * h_kv * p.all_rows * (d + 2) * sizeof(float));
    return p;
}

hipError_t launch_attention_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const void *pages, const AttnQ4Plan &p, void *workspace, void *out, int num_cus,
                               hipStream_t st) {
    char *ws = static_cast<char *>(workspace);
    AttnQ4Args a = {};
    a.q = static_cast<const _Float16 *>(q);
    a.out = static_cast<_Float16 *>(out);
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv;
    a.workers = p.workers, a.least = p.least, a.whole = p.shared ? 0 : kWhole;  // (no second launch: nothing is cut)
    a.ws_o = reinterpret_cast<float *>(ws + p.partial);
    a.ws_ml = a.ws_o + (size_t)p.workers * 2 * 16 * d;
    a.scale = 1.4426950408889634f / sqrtf((float)d);
    ManyArgs many = {};
    _Float16 *kc = nullptr, *vc = nullptr;
    if (p.slots > 0) {
        a.plan = reinterpret_cast<int *>(ws + p.plan);
        kc = reinterpret_cast<_Float16 *>(ws + p.copies);
        vc = kc + (size_t)p.slots * h_kv * p.pages * kPage * d;
        many.req = req;
        many.plan = a.plan;
        many.pages = a.pages;
        many.kc = kc, many.vc = vc;
        many.g = a.g, many.h_kv = h_kv, many.slots = p.slots, many.records = p.records, many.block_rows = 128 / p.shares, many.chunk_steps = p.chunk_steps;
        many.max_pages = p.pages, many.few = few_rows(p.all_rows);
    }
    hipError_t e = hipErrorInvalidValue;
    switch (d) {
        case 64: e = launch<64>(a, many, p, num_cus, st); break;
        case 128: e = launch<128>(a, many, p, num_cus, st); break;
        case 256: e = launch<256>(a, many, p, num_cus, st); break;
    }
    if (e != hipSuccess || p.slots == 0) return e;
    return launch_attention_many(q, kc, vc, h_q, h_kv, d, p.pages * kPage, a.plan, p.records, p.shares, p.items, p.all_rows,
                                 p.chunk_steps > 0 ? reinterpret_cast<float *>(ws + p.many_partial) : nullptr, out, st);
}

}  // namespace qfc
