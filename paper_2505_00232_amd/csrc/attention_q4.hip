// Attention of the new tokens of a batch of requests over their paged 4-bit cache: how the pages are dealt to wavefronts, and how partial results are joined.  What a wavefront does with
// a page: attention_q4_rows.h.
#include "attention_q4_rows.h"

namespace qfc {
namespace {

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

// (Sums of places: requests whose arrays overlap may have more of them than a call's limits allow.  What lies behind those, AttnQ4Args::most, 2^24 and more below the largest int, so
// that no place of a unit that is worked on passes it, is left out.)
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

// Up to 16 query rows of a KV head at a time.  The wavefronts work for themselves, each with copies of its own on the way.  Bound: memory where rows are few (32 requests of up to 8192
// positions, 32 heads on 8 of 128 values: 168 MB in 41 us, 4.1 TB/s), the some 450 vector instructions of a page and block, and little that runs beside them, where they are many
// (prompts of 1024 and 601 tokens 72 us).  Two blocks that share the codes' taking apart need more registers than two wavefronts of a SIMD have, and were slower (prompts 187 us, 167
// with one, both before blocks came in pairs).
template <int D>
__global__ __launch_bounds__(256, kWgs) void attn_q4_kernel(AttnQ4Args a) {
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Rows<D> rows16(lds, wave, lane);
    const int m = rows16.m, r = rows16.r;
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
        const int ahead = numbers(0);

        // ---- queries
        const bool real = row0 + m < rows;
        const int token = real ? (row0 + m) / a.g : 0, head = kv * a.g + (real ? (row0 + m) % a.g : 0);
        const size_t at = ((size_t)(span.first + token) * a.h_q + head) * D;
        const int lim = real ? n - span.count + token + 1 : 0;  // positions the lane's row sees (none where 0 or less)
        rows16.load(a.q + at, real, a.scale);
        rows16.walk(count, lim, n, a.pages, a.h_kv, kv, ahead, numbers, [&](int i) __attribute__((always_inline)) { return (page0 + i) * kPage; });

        // ---- output row m (2^kFactor times, unnormalized), its maximum and sum
        const float sum = rows16.sum(), inv = sum != 0.0f ? 1.0f / sum : 0.0f;  // (a row that sees nothing: 0; one of a NaN stays NaN)
        const size_t part = partial_of(unit, worker, units.share) * 16 + m;
        rows16.columns([&](int d, const v4f &o) __attribute__((always_inline)) {
            if (!real) return;
            if (whole)
                *reinterpret_cast<h4 *>(a.out + at + d) = h4{(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
            else
                *reinterpret_cast<v4f *>(a.ws_o + part * D + d) = o;
        });
        if (real && !whole && r == 0) {
            a.ws_ml[part * 2] = rows16.run_max;
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
