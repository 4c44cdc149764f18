// Attention over the paged 4-bit cache in parts that are joined afterwards: of requests whose first positions are the same pages, and over selected pages.
//
// A part is a run of pages and 16 query rows of a KV head; it leaves unnormalized outputs o, a maximum m and a sum l, and
//   out = sum_i e^(m_i - m) o_i / sum_i e^(m_i - m) l_i,   m = max_i m_i.
// The rows of a group of requests meet their common pages as rows of one request do, whatever request they are of: what the pages cost is shared by 16 rows.  What a wavefront does with a
// page, and in which precision: attention_q4_rows.h.
#include "attention_q4_rows.h"

namespace qfc {
namespace {

struct PartsArgs {
    const _Float16 *q;  // [tokens, h_q, D]
    _Float16 *out;
    const char *pages;
    Requests req;
    const int *group_start, *prefix;  // of groups with common pages
    int groups, group_tokens, longest;
    float *ws_o, *ws_ml;  // [slots][tokens * h_q][D] partial outputs, [..][2] (maximum, sum; 0: nothing was seen, no output)
    int h_q, h_kv, g;
    int prefix_parts, parts;  // slots: of common pages, and behind them of the others
    long prefix_items, items;  // of workgroups; items: all of them
    bool wide;
    float scale;
};

// x among runs of len(i) places, i = 0, 1, .. count - 1: which run, and the place in it (-1: behind the last).  A lane looks at one run at a time.
struct Found {
    int run, place;
};
template <class Len>
__device__ __forceinline__ Found find(int x, int count, int lane, const Len &len) {
    for (int c = 0; c < count; c += 64) {
        const int mine = c + lane < count ? len(c + lane) : 0, upto = sum_upto(mine);
        const uint64_t past = __ballot(upto > x);
        if (past) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
            const int len_of = __builtin_amdgcn_readlane(mine, l), place = x - (__builtin_amdgcn_readlane(upto, l) - len_of);
            return place < len_of ? Found{c + l, place} : Found{-1, 0};  // (sums that ended at the largest int)
        }
        x -= __builtin_amdgcn_readlane(upto, 63);
    }
    return Found{-1, 0};
}

// Requests of group i, their rows, and the pages in front of all their new tokens that they have in common
struct Group {
    int lead, pages;  // the first one with tokens: its table's row is read
};
__device__ __forceinline__ int group_end(const PartsArgs &a, int i) { return min(max(a.group_start[i], 0), a.req.batch); }
__device__ __forceinline__ int token_at(const Requests &q, int b) { return min(max(q.start[b], 0), q.tokens); }
__device__ __forceinline__ int tokens_of_group(const PartsArgs &a, int i) {
    return min(max(token_at(a.req, group_end(a, i + 1)) - token_at(a.req, group_end(a, i)), 0), a.group_tokens);
}
__device__ __forceinline__ Group group_of(const PartsArgs &a, int i, int lane) {
    const int first = group_end(a, i), end = group_end(a, i + 1);
    int least = min(max(a.prefix[i], 0), a.longest), lead = INT32_MAX;
#pragma unroll 4
    for (int b0 = first; b0 < end; b0 += 64) {  // (no look at other lanes in here: several rounds' loads are on their way at once)
        const int b = min(b0 + lane, end - 1);
        const Span s = span_of(a.req, b);
        if (s.count > 0) least = min(least, max(s.positions - s.count, 0)), lead = min(lead, b);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) least = min(least, __shfl_xor(least, off, 64)), lead = min(lead, __shfl_xor(lead, off, 64));
    return Group{__builtin_amdgcn_readfirstlane(lead == INT32_MAX ? 0 : lead), __builtin_amdgcn_readfirstlane(lead == INT32_MAX ? 0 : least / kPage)};
}

// The wavefronts of a workgroup have an equal share each of the same rows' pages and meet in LDS, in the places of their pages.
template <int D, bool SPREAD = false, int WAVES = 4>
struct Meeting {
    // A thread (of the first 256) has columns of row threadIdx.x / 16: of all D from 4 (threadIdx.x % 16) on 4, and every 64th behind them; SPREAD: 2 of the row's group
    static constexpr int PER = SPREAD ? 2 : 4;
    typedef float cols __attribute__((ext_vector_type(PER)));
    static constexpr int STRIDE = D + 4;  // of a row (banks)
    static constexpr int WAVE = 2 * Place<D>::PART / 4;
    static_assert(16 * (STRIDE + 2) <= WAVE, "a wavefront's partial outputs, maxima and sums take its pages' places");
    float *const lds;  // (nothing beside it: with heads of 256 values two workgroups take a compute unit's LDS to the last byte)
    __device__ __forceinline__ float *sums_of(int wave, int row) const { return lds + wave * WAVE + 16 * STRIDE + 2 * row; }
    // put(column, output, 1 / sum) for the thread's columns, then put_sum(maximum, sum).
    // What a lane knows of row m the threads of row threadIdx.x / 16 ask for: theirs(x).
    template <class T>
    __device__ static __forceinline__ T theirs(T x) {
        return __shfl(x, (int)(threadIdx.x >> 4), 64);
    }
    template <class Put, class PutSum>
    __device__ __forceinline__ void meet(const Rows<D, SPREAD> &rows, int wave, bool wanted, const Put &put, const PutSum &put_sum) const {
        float *const mine = lds + wave * WAVE + rows.m * STRIDE;
        rows.columns([&](int d, const v4f &o) __attribute__((always_inline)) { *reinterpret_cast<v4f *>(mine + d) = o; });
        const float own_sum = rows.sum();
        if (rows.r == 0) sums_of(wave, rows.m)[0] = rows.run_max, sums_of(wave, rows.m)[1] = own_sum;
        __syncthreads();
        if (wanted && threadIdx.x < 256) {
            const int row = threadIdx.x >> 4;
            float f[WAVES], top = sums_of(0, row)[0], l = 0.0f;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sums_of(w, row)[0]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                f[w] = __builtin_amdgcn_exp2f(sums_of(w, row)[0] - top);
                l = fmaf(f[w], sums_of(w, row)[1], l);
            }
            const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
            for (int c = 0; c < (SPREAD ? 1 : D / 64); ++c) {
                const int d = SPREAD ? row / Rows<D, SPREAD>::ROWS * 32 + 2 * (threadIdx.x & 15) : 64 * c + 4 * (threadIdx.x & 15);
                cols o = {};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const cols x = *reinterpret_cast<const cols *>(lds + w * WAVE + row * STRIDE + d);
#pragma unroll
                    for (int i = 0; i < PER; ++i) o[i] = fmaf(f[w], x[i], o[i]);
                }
                put(d, o, inv);
            }
            if ((threadIdx.x & 15) == 0) put_sum(top, l);
        }
        __syncthreads();
    }
};
__device__ __forceinline__ h4 rounded(const v4f &o, float by) { return h4{(_Float16)(o[0] * by), (_Float16)(o[1] * by), (_Float16)(o[2] * by), (_Float16)(o[3] * by)}; }
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ h2 rounded(const v2f &o, float by) { return h2{(_Float16)(o[0] * by), (_Float16)(o[1] * by)}; }

// Sums over parts, eight on their way at a time: part i is at place(i), its maximum and sum at ml, its columns at o
template <class Place>
__device__ __forceinline__ v4f joined(const float *ml, const float *o_at, int stride, int parts, const Place &place, float &inv) {
    float top = kNothingYet, l = 0.0f;
    v4f o = {};
    for (int s0 = 0; s0 < parts; s0 += 8) {
        float ms[8], ls[8];
        v4f os[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const size_t at = place(min(s0 + i, parts - 1));
            ms[i] = ml[at * 2], ls[i] = ml[at * 2 + 1];
            os[i] = *reinterpret_cast<const v4f *>(o_at + at * stride);
        }
        float new_top = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (s0 + i >= parts) ls[i] = 0.0f;
            new_top = ls[i] != 0.0f ? fmaxf(new_top, ms[i]) : new_top;
        }
        const float corr = __builtin_amdgcn_exp2f(top - new_top);
        top = new_top, l *= corr;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= corr;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (ls[i] == 0.0f) continue;  // (nothing was seen: what stands there is not defined)
            const float f = __builtin_amdgcn_exp2f(ms[i] - top);
            l = fmaf(f, ls[i], l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, os[i][e], o[e]);
        }
    }
    inv = l != 0.0f ? 1.0f / l : 0.0f;
    return o;
}

// ---- selected pages.  Units of a token, a KV head and 16 of its query heads, one behind the other, each with the `count` places of its list; every workgroup has `share` places in a row, whatever
// units they are of.  Of a unit that several have a part of, each leaves partial results: two at most per workgroup, of the unit that its share begins inside of (or with), and of the one
// that it ends inside of.
struct SelectedArgs {
    const _Float16 *q;
    _Float16 *out;
    const char *pages;
    Requests req;
    const int *selected;  // [tokens, h_kv, count]
    float *ws_o, *ws_ml;  // [workgroups][2][16][D], [..][2]
    int h_q, h_kv, g, head_blocks, count, waves;
    long share, places;
    float scale;
};
struct Unit {
    long begin, end;
    int token, kv, head0;
};
__device__ __forceinline__ Unit unit_of(const SelectedArgs &a, long place) {
    Unit u;
    const long unit = place / a.count, block = unit / a.h_kv;
    u.begin = unit * a.count, u.end = u.begin + a.count;
    u.kv = (int)(unit % a.h_kv), u.head0 = (int)(block % a.head_blocks) * 16, u.token = (int)(block / a.head_blocks);
    return u;
}

constexpr float kNobodys = -1.0f;  // sum of the parts of a row that is left as it was

template <int D, bool SPREAD, int WAVES>
__global__ __launch_bounds__(64 * WAVES, kWgs) void attn_q4_selected_kernel(SelectedArgs a) {
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    typedef Meeting<D, SPREAD, WAVES> F;
    Rows<D, SPREAD> rows(lds, wave, lane);
    const F four = {lds};
    const long from = blockIdx.x * a.share, stop = min(from + a.share, a.places);
    for (long x = from; x < stop;) {
        const Unit u = unit_of(a, x);
        const long last = min(stop, u.end);
        const int p0 = (int)(x - u.begin), p1 = (int)(last - u.begin);
        const bool whole = p0 == 0 && last == u.end;
        const size_t part0 = ((size_t)blockIdx.x * 2 + (u.begin > from ? 1 : 0)) * 16;
        x = last;
        const int *const list = a.selected + ((size_t)u.token * a.h_kv + u.kv) * a.count;
        const int begin = p0 + (int)((long)(p1 - p0) * wave / WAVES), count = __builtin_amdgcn_readfirstlane(p0 + (int)((long)(p1 - p0) * (wave + 1) / WAVES) - begin);
        int place = lane < count ? list[begin + lane] : -1;  // of the page in its request, a page per lane; on its way before anything is known of the request
        Span span;
        const int b = __builtin_amdgcn_readfirstlane(request_of_token(a.req, u.token, lane, span));
        if (b >= a.req.batch || u.token < span.first || u.token - span.first >= span.count) {  // nobody's
            if (!whole && threadIdx.x < 16) a.ws_ml[(part0 + threadIdx.x) * 2 + 1] = kNobodys;
            continue;
        }
        const int n = span.positions, lim = n - span.count + u.token - span.first + 1;
        const bool real = u.head0 + rows.row() < a.g;
        const int head = u.kv * a.g + min(u.head0 + rows.row(), a.g - 1);
        const size_t at = (size_t)u.token * a.h_q + head;
        auto page_at = [&](int of) __attribute__((always_inline)) { return of >= 0 && of < (a.req.max_context + kPage - 1) / kPage ? page_of(a.req, b, of * kPage) : -1; };
        auto numbers = [&](int i) __attribute__((always_inline)) {
            place = i + lane < count ? list[begin + i + lane] : -1;
            return page_at(place);
        };
        const int ahead = page_at(place);
        rows.load(a.q + at * D, real, a.scale);
        rows.walk(count, real ? lim : 0, n, a.pages, a.h_kv, u.kv, ahead, numbers,
                  [&](int i) __attribute__((always_inline)) { return (int)((uint32_t)__builtin_amdgcn_readlane(place, i & 63) * kPage); });
        const size_t their_at = F::theirs((unsigned long long)at), part = part0 + (threadIdx.x >> 4);
        four.meet(
            rows, wave, F::theirs((int)real) != 0,
            [&](int d, const typename F::cols &o, float inv) __attribute__((always_inline)) {
                if (whole)
                    *reinterpret_cast<decltype(rounded(o, inv)) *>(a.out + their_at * D + d) = rounded(o, inv);
                else
                    *reinterpret_cast<typename F::cols *>(a.ws_o + part * D + d) = o;
            },
            [&](float top, float l) __attribute__((always_inline)) {
                if (!whole) a.ws_ml[part * 2] = top, a.ws_ml[part * 2 + 1] = l;
            });
    }
}

// A workgroup for the unit that the share of workgroup blockIdx.x + 1 begins inside of, if that is the first to do so; D / 4 threads per row
template <int D, bool SPREAD>
__global__ __launch_bounds__(256) void attn_q4_join_selected_kernel(SelectedArgs a) {
    const int d = 4 * (threadIdx.x % (D / 4));
    const long x = ((long)blockIdx.x + 1) * a.share;
    const Unit u = unit_of(a, x);
    if (u.begin >= x || x - u.begin > a.share) return;
    const long w0 = u.begin / a.share;
    const int parts = (int)((u.end - 1) / a.share - w0) + 1;
    for (int row = threadIdx.x / (D / 4); row < min(16, a.g - u.head0); row += 1024 / D) {
        const int held = SPREAD ? d / 32 * Rows<D, SPREAD>::ROWS + row : row;  // (the row of the parts that has these columns)
        float inv;
        auto place = [&](int c) __attribute__((always_inline)) { return (size_t)((w0 + c) * 2 + (c == 0 && u.begin > w0 * a.share ? 1 : 0)) * 16 + held; };
        const float first = a.ws_ml[place(0) * 2 + 1];
        const v4f o = joined(a.ws_ml, a.ws_o + d, D, parts, place, inv);
        if (first != kNobodys) *reinterpret_cast<h4 *>(a.out + ((size_t)u.token * a.h_q + u.kv * a.g + u.head0 + row) * D + d) = rounded(o, inv);
    }
}

// ---- common pages of many rows.  What attention_q4_rows.h does to a page for 16 query rows, most of its instructions, is to take its codes apart: 551 vector instructions of a page and 16 rows,
// of which 192 for that.  Here the four wavefronts of a workgroup take a page's codes apart once, into LDS as binary16 whole numbers code - 8 (exact, as are the products with the queries), and
// multiply them with 32 rows each (342 instructions of a page and 16 rows); steps, offsets and P are taken into the sums in the same way and with the same precision as there, steps of 2 and
// more in a turn of their own (where every page has some: 1024 rows behind 20011 positions 214 -> 355 us):
//   q . k = sum_j step_j (q_j . (code_j - 8)) + sum_j offset_j sum q_j,   out_d = sum_p (p step_j) (code - 8) + sum_p p offset_j
// The common pages are in front of all rows' positions: nothing is masked.  Bound: the LDS, 63 reads of a KiB of a page and wavefront at 64 bytes a cycle, beside vector instructions in 71 % of the
// cycles (1024 rows of 8 heads of 128 values behind 20000 positions 173 us: 485 TFLOP/s).
template <int D>
struct Wide {
    typedef PageLayout<D> L;
    static constexpr int G = L::G, W = L::W, DT = D / 16, NB = 2, ROWS = 64 * NB;
    // LDS: K operands [4 tiles][G][64 lanes], V operands [G][low, high][2 halves of 16 positions][64 lanes], 16 bytes each; then the page's steps and offsets of keys, and of values: steps below 2
    // (zeros for the others), offsets, steps of 2 and more (zeros for the others)
    static constexpr int kV = 128 * D, kHeadK = 256 * D, kHeadV = 264 * D, kBytes = 276 * D;
    static constexpr int kStepK = kHeadK, kOffsetK = kHeadK + 4 * D, kStepV = kHeadV, kOffsetV = kHeadV + 4 * D, kLargeV = kHeadV + 8 * D;
    // A page on its way: what a thread has of it
    static constexpr int kPiecesK = 4 * (G / W) * 64, kPiecesV = G * 64, PK = (kPiecesK + 255) / 256, PV = (kPiecesV + 255) / 256;
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    words k[PK];
    u32x4 v[PV], head;
    __device__ __forceinline__ void fetch(const char *page) {
#pragma unroll
        for (int i = 0; i < PK; ++i) k[i] = *reinterpret_cast<const words *>(page + L::kCodesK + (256 * i + (int)threadIdx.x) * (4 * W));
#pragma unroll
        for (int i = 0; i < PV; ++i) v[i] = *reinterpret_cast<const u32x4 *>(page + L::kCodesV + min(256 * i + (int)threadIdx.x, kPiecesV - 1) * 16);
        const int piece = min((int)threadIdx.x, D - 1);  // D / 2 pieces of 16 bytes of keys' steps and offsets, then of values'
        head = *reinterpret_cast<const u32x4 *>(page + (piece < D / 2 ? L::kStepK + piece * 16 : L::kStepV + (piece - D / 2) * 16));
    }
    // two codes, 16 bits apart, as binary16 code - 8
    __device__ static __forceinline__ uint32_t two(uint32_t w) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 x = __builtin_bit_cast(h2, __builtin_amdgcn_bitop3_b32(w, 0x000F000Fu, 0x64006400u, 0xEA));  // 1024 + code
        return __builtin_bit_cast(uint32_t, x - h2{(_Float16)1032.0f, (_Float16)1032.0f});
    }
    __device__ __forceinline__ void put(char *lds) const {
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int piece = 256 * i + (int)threadIdx.x, lane = piece % 64, tile = piece / 64 / (G / W), j0 = piece / 64 % (G / W) * W;
#pragma unroll
            for (int w = 0; w < W; ++w) *reinterpret_cast<u32x4 *>(lds + ((tile * G + j0 + w) * 64 + lane) * 16) = u32x4{two(k[i][w]), two(k[i][w] >> 4), two(k[i][w] >> 8), two(k[i][w] >> 12)};
        }
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            const int piece = 256 * i + (int)threadIdx.x, lane = piece % 64, j = piece / 64;
            if (kPiecesV % 256 != 0 && piece >= kPiecesV) break;
#pragma unroll
            for (int high = 0; high < 2; ++high)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t a = v[i][2 * u] >> (4 * high), b = v[i][2 * u + 1] >> (4 * high);
                    *reinterpret_cast<u32x4 *>(lds + kV + (((j * 2 + high) * 2 + u) * 64 + lane) * 16) = u32x4{two(a), two(a >> 8), two(b), two(b >> 8)};
                }
        }
        const int piece = (int)threadIdx.x;
        if (piece >= D) return;
        u32x4 large = {};
        if (piece >= D / 2 && piece < D / 2 + D / 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) large[i] = head[i] & (head[i] >> 14 & 0x00010001u) * 0xFFFFu;  // (exponents from 2.0's on)
            *reinterpret_cast<u32x4 *>(lds + kLargeV + (piece - D / 2) * 16) = large;
        }
        *reinterpret_cast<u32x4 *>(lds + kHeadK + piece * 16) = head & ~large;
    }
};

// The state of NB blocks of 16 rows, lane (m, r) as in Rows
template <int D>
struct WideRows {
    typedef Wide<D> S;
    static constexpr int G = S::G, DT = S::DT, NB = S::NB;
    const int lane, m, r;
    h8 qf[NB][G], sums[NB];
    float to_score[NB], run_max[NB];
    v4f acc[NB][DT], rest[NB];
    // The maximum may be kLag below a score (in units of log 2): what hardly moves it costs no pass over the sums.  P is taken 2^kAt times as large, at most 2^14.5 then, and its products with
    // steps below 2 are below 2^15.5: binary16 keeps as many bits of small ones as in attention_q4_rows.h.  (1024 rows behind 20011 positions 214 us with all that is behind them; with a lag of 2
    // and P a quarter as large 209.)
    static constexpr float kLag = 0.5f, kAt = kFactor;
    static_assert(kAt + kLag + 1.0f <= 15.5f, "binary16 holds 2^16: a part of it is for what scores of thousands are rounded by");
    __device__ __forceinline__ WideRows(int l) : lane(l), m(l & 15), r(l >> 4) {}

    __device__ __forceinline__ void load(int nb, const _Float16 *q, bool real, float scale) {
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const h8 zero = {};
            qf[nb][j] = real ? *reinterpret_cast<const h8 *>(q + 32 * j + 8 * r) : zero;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)qf[nb][j][e]));
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        // the largest to 2^9 .. 2^10: 32 of them add up to what binary16 holds, and what it loses of the smallest is 2^-34 of the largest
        const int up = top > 0.0f ? 10 - __builtin_amdgcn_frexp_expf(top) : 0;
        const float up2 = __builtin_amdgcn_ldexpf(1.0f, up);
        to_score[nb] = __builtin_amdgcn_ldexpf(scale, -up);
        sums[nb] = h8{};
#pragma unroll
        for (int j = 0; j < G; ++j) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = (float)qf[nb][j][e] * up2;
                s += x;
                qf[nb][j][e] = (_Float16)x;
            }
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            const _Float16 hi = (_Float16)s, lo = (_Float16)(s - (float)hi);
            sums[nb][j] = r == 0 ? hi : r == 1 ? lo : (_Float16)0.0f;
        }
        run_max[nb] = kNothingYet;
        rest[nb] = v4f{};
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[nb][t] = v4f{};
    }

    typedef __attribute__((address_space(3))) const char *Lds;
    template <class T>
    __device__ static __forceinline__ T read(Lds at) {
        return *reinterpret_cast<__attribute__((address_space(3))) const T *>(at);
    }
    // The operands of a lane are at constant distances from four addresses.  (Nothing says so to the compiler but that it does not know the four: it kept some hundred sums in registers otherwise, from
    // page to page, and had to spill.)
    Lds at16, at_r, at_m, at_rows, at_lane;
    __device__ __forceinline__ void page(const char *lds) {
        const Lds base = (Lds)lds;
        at16 = base + 16 * lane, at_r = base + 32 * r, at_m = base + 2 * G * m, at_rows = base + min(m, G - 1) * (2 * kPage) + 32 * r, at_lane = base + 4 * lane;
        asm volatile("" : "+v"(at16), "+v"(at_r), "+v"(at_m), "+v"(at_rows), "+v"(at_lane));
        // ---- scores; lane (m, r), element 4 t + i: position 16 r + 4 t + i
        float sc[NB][16];
        {
            v4f part[NB][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                typedef _Float16 offsets __attribute__((ext_vector_type(G)));
                const offsets x = read<offsets>(at_m + S::kOffsetK + 32 * G * t);  // (whatever r: the sums of q are 0 behind the first two)
                h8 off = {};
#pragma unroll
                for (int j = 0; j < G; ++j) off[j] = x[j];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) part[nb][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, sums[nb], v4f{}, 0, 0, 0);
            }
            // (operands of a group are asked for while the one before is worked on)
            h8 op[2][4], st[2][2];
            auto ask = [&](int j) __attribute__((always_inline)) {
                st[j & 1][0] = read<h8>(at_r + S::kStepK + j * kPage * 2), st[j & 1][1] = read<h8>(at_r + S::kStepK + j * kPage * 2 + 16);
#pragma unroll
                for (int t = 0; t < 4; ++t) op[j & 1][t] = read<h8>(at16 + (t * G + j) * 1024);
            };
            ask(0);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                if (j + 1 < G) ask(j + 1);
                v4f x[NB][4];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) x[nb][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op[j & 1][t], qf[nb][j], v4f{}, 0, 0, 0);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[nb][t][i] = fmaf((float)st[j & 1][t >> 1][4 * (t & 1) + i], x[nb][t][i], part[nb][t][i]);
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[nb][e] = part[nb][e >> 2][e & 3];
        }
        // ---- P, 2^kAt times as large
        // (one branch for all blocks: behind a branch for the first, the compiler put off the sums of the second and kept every product that they are made of)
        h8 pv[NB][2];
        float most[NB];
        bool more = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            most[nb] = fmaxf(sc[nb][0], sc[nb][1]);
#pragma unroll
            for (int e = 2; e < 16; e += 2) most[nb] = fmaxf(fmaxf(most[nb], sc[nb][e]), sc[nb][e + 1]);
            most[nb] = over_rows(most[nb]) * to_score[nb];
            more = more || most[nb] > run_max[nb] + kLag;
        }
        if (__any(more)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float new_max = fmaxf(run_max[nb], most[nb]), corr = __builtin_amdgcn_exp2f(run_max[nb] - new_max);
                run_max[nb] = new_max;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) acc[nb][t][i] *= corr;
                    rest[nb][i] *= corr;
                }
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float from_max = kAt - run_max[nb];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[nb][e] = __builtin_amdgcn_exp2f(fmaf(sc[nb][e], to_score[nb], from_max));
                pv[nb][e >> 3][e & 7] = (_Float16)sc[nb][e];
            }
        }
        // ---- second product
#pragma unroll
        for (int u = 0; u < 2; ++u) {  // rows 0 .. G - 1: offsets; row 15: ones; the others are not used
            const u32x4 w = read<u32x4>(at_rows + S::kOffsetV + 16 * u);
            const u32x4 rows = {m == 15 ? 0x3C003C00u : w.x, m == 15 ? 0x3C003C00u : w.y, m == 15 ? 0x3C003C00u : w.z, m == 15 ? 0x3C003C00u : w.w};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) rest[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, rows), pv[nb][u], rest[nb], 0, 0, 0);
        }
        // Steps below 2; those of 2 and more in a turn of their own behind it, with each row's P lowered until its largest product with one of them is below 2^15 (by powers of two: exact in P and in
        // sums of 32 bits): what binary16 then loses is little against a product that is in the row's sums, and the small steps, in this page and the others, keep their bits.
        auto product = [&](Lds steps) __attribute__((always_inline)) {
            h8 step[2], lo[2], hi[2];
            auto ask = [&](int k) __attribute__((always_inline)) {
                const int j = k / 2, u = k % 2;
                step[u] = read<h8>(steps + j * kPage * 2 + 16 * u), lo[u] = read<h8>(at16 + S::kV + (4 * j + u) * 1024), hi[u] = read<h8>(at16 + S::kV + (4 * j + 2 + u) * 1024);
            };
            ask(0);
#pragma unroll
            for (int k = 0; k < 2 * G; ++k) {
                const int j = k / 2, u = k % 2;
                __builtin_amdgcn_sched_barrier(0);  // (one after the other: registers)
                if (k + 1 < 2 * G) ask(k + 1);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    h8 p;
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = (_Float16)fmaf(sc[nb][8 * u + e], (float)step[u][e], 0.0f);  // (with the sum one instruction takes 32 and 16 bits)
                    acc[nb][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[u], p, acc[nb][2 * j], 0, 0, 0);
                    acc[nb][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[u], p, acc[nb][2 * j + 1], 0, 0, 0);
                }
            }
        };
        product(at_r + S::kStepV);
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < G; j += 2) bits |= read<uint32_t>(at_lane + S::kLargeV + j * kPage * 2);  // (two groups' steps are 64 dwords)
        if (__any(bits != 0)) {
            float back[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float most = 0.0f;
#pragma unroll
                for (int k = 0; k < 2 * G; ++k) {
                    __builtin_amdgcn_sched_barrier(0);
                    const h8 step = read<h8>(at_r + S::kLargeV + k / 2 * kPage * 2 + 16 * (k % 2));
#pragma unroll
                    for (int e = 0; e < 8; ++e) most = fmaxf(most, sc[nb][8 * (k % 2) + e] * (float)step[e]);
                }
                most = over_rows(most);
                const int down = most >= 32768.0f ? __builtin_amdgcn_frexp_expf(most) - 15 : 0;
                const float by = __builtin_amdgcn_ldexpf(1.0f, -down);
                back[nb] = __builtin_amdgcn_ldexpf(1.0f, down);
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[nb][e] *= by;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nb][t][i] *= by;
            }
            Lds again = at_r + S::kLargeV;
            asm volatile("" : "+v"(again));  // (steps are read twice rather than kept)
            product(again);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nb][t][i] *= back[nb];
        }
    }
    __device__ __forceinline__ float sum(int nb) const { return __shfl(rest[nb][3], 48 + m, 64); }
    template <class Put>
    __device__ __forceinline__ void columns(int nb, const Put &put) const {
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const float off = __shfl(rest[nb][j & 3], (j >> 2) * 16 + m, 64);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                v4f o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = acc[nb][2 * j + k][i] + off;
                put(32 * j + 16 * k + 4 * r, o);
            }
        }
    }
};

// A workgroup per part of 64 NB rows of a group.  (A kernel of its own: beside the other path's state it had no registers for loads that are ahead of their use.)
template <int D>
__global__ __launch_bounds__(256, 2) void attn_q4_wide_kernel(PartsArgs a) {
    typedef Wide<D> S;
    constexpr int NB = S::NB;
    extern __shared__ char wide_lds[];
    char *const lds = wide_lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = (int)(blockIdx.x % a.h_kv), part = (int)(blockIdx.x / a.h_kv % a.prefix_parts), block = (int)(blockIdx.x / a.h_kv / a.prefix_parts);
    const Found f = find(block, a.groups, lane, [&](int i) __attribute__((always_inline)) { return (int)(((long)tokens_of_group(a, i) * a.g + S::ROWS - 1) / S::ROWS); });
    if (f.run < 0) return;
    const Group group = group_of(a, f.run, lane);
    const int first = token_at(a.req, group_end(a, f.run)), rows_all = tokens_of_group(a, f.run) * a.g;
    const long all_rows = (long)a.req.tokens * a.h_q;
    const int per = max(1, (group.pages + a.prefix_parts - 1) / a.prefix_parts), from = min(part * per, group.pages), to = min(from + per, group.pages);
    WideRows<D> rows(lane);
    size_t out_row[NB];
    bool real[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int row = f.place * S::ROWS + (wave * NB + nb) * 16 + rows.m, held = min(row, rows_all - 1);
        real[nb] = row < rows_all;
        const size_t at = (size_t)(first + held / a.g) * a.h_q + kv * a.g + held % a.g;
        out_row[nb] = (size_t)part * all_rows + at;
        if (from < to) rows.load(nb, a.q + at * D, real[nb], a.scale);
        if (from >= to && rows.r == 0 && real[nb]) a.ws_ml[out_row[nb] * 2 + 1] = 0.0f;
    }
    if (from >= to) return;
    // the next page that there is, from place i on; a lane knows one of 64 places
    int numbers = -1, known = from - 64;
    auto following = [&](int &i) __attribute__((always_inline)) {
        for (;; ++i) {
            if (i >= to) return -1;
            if (i >= known + 64) {
                known = i;
                numbers = i + lane < to ? page_of(a.req, group.lead, (i + lane) * kPage) : -1;
            }
            const int page = __builtin_amdgcn_readlane(numbers, i - known);
            if (page >= 0) return page;
        }
    };
    int i = from, page = following(i);
    S raw;
    auto fetch = [&](int of) __attribute__((always_inline)) { raw.fetch(a.pages + ((size_t)of * a.h_kv + kv) * PageLayout<D>::kBytes); };
    if (page >= 0) fetch(page);
    // (the next page is taken apart into the other place: one barrier per page)
    char *now = lds, *other = lds + S::kBytes;
    if (page >= 0) {
        raw.put(now);
        ++i;
        page = following(i);
        if (page >= 0) fetch(page);
        for (;;) {
            __syncthreads();
            rows.page(now);
            if (page < 0) break;
            raw.put(other);
            ++i;
            page = following(i);
            if (page >= 0) fetch(page);
            char *const x = now;
            now = other, other = x;
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float l = rows.sum(nb);
        if (!real[nb]) continue;
        rows.columns(nb, [&](int d, const v4f &o) __attribute__((always_inline)) { *reinterpret_cast<v4f *>(a.ws_o + out_row[nb] * D + d) = o; });
        if (rows.r == 0) a.ws_ml[out_row[nb] * 2] = rows.run_max[nb], a.ws_ml[out_row[nb] * 2 + 1] = l;
    }
}

// ---- common pages.  A workgroup per part of the rows of a group or a request.
template <int D>
__global__ __launch_bounds__(256, D <= 128 ? 3 : kWgs) void attn_q4_parts_kernel(PartsArgs a) {
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long all_rows = (long)a.req.tokens * a.h_q;
    Rows<D> rows(lds, wave, lane);
    const Meeting<D> four = {lds};
    const int m = rows.m;
    for (long item = blockIdx.x; item < a.items; item += gridDim.x) {
        // ---- which rows, which pages: from .. to - 1 of request b
        int b, lim, n, from, first, row, rows_all, pages;
        const bool common = item < a.prefix_items;
        const long x = common ? item : item - a.prefix_items;
        const int parts = common ? a.prefix_parts : a.parts, kv = (int)(x % a.h_kv), part = (int)(x / a.h_kv % parts), block = (int)(x / a.h_kv / parts);
        if (common) {
            const Found f = find(block, a.groups, lane, [&](int i) __attribute__((always_inline)) { return (int)(((long)tokens_of_group(a, i) * a.g + 15) / 16); });
            if (f.run < 0) {  // (on to the items behind the groups')
                item += (a.prefix_items - 1 - item) / gridDim.x * gridDim.x;
                continue;
            }
            const Group group = group_of(a, f.run, lane);
            b = group.lead, pages = group.pages;
            first = token_at(a.req, group_end(a, f.run)), rows_all = tokens_of_group(a, f.run) * a.g, row = f.place * 16 + m;
            n = pages * kPage, lim = n, from = 0;
        } else {
            Found f = {block, 0};
            if (a.req.max_tokens * a.g > 16)
                f = find(block, a.req.batch, lane, [&](int i) __attribute__((always_inline)) { return (span_of(a.req, i).count * a.g + 15) / 16; });
            if (f.run < 0 || f.run >= a.req.batch) return;
            b = f.run;
            const Span s = span_of(a.req, b);
            first = s.first, rows_all = s.count * a.g, row = f.place * 16 + m;
            n = s.positions, lim = n - s.count + row / a.g + 1;
            // its group, and the pages that are done with that
            int before = 0;
            for (int c = 0; c <= a.groups; c += 64) before += __popcll(__ballot(c + lane <= a.groups && group_end(a, min(c + lane, a.groups)) <= b));
            from = before > 0 && before <= a.groups ? group_of(a, before - 1, lane).pages : 0;
            // (the last row's positions are the most)
            const int sees = max(0, n - s.count + min(f.place * 16 + 15, rows_all - 1) / a.g + 1);
            pages = (sees + kPage - 1) / kPage;
        }
        if (rows_all <= 0) continue;
        const bool real = row < rows_all;
        row = min(row, rows_all - 1);
        const int token = first + row / a.g, head = kv * a.g + row % a.g, slot = part + (common ? 0 : a.prefix_parts);
        const int per = max(4, (max(pages - from, 0) + parts - 1) / parts);
        from = min(from + part * per, max(pages, from));
        const int to = min(from + per, max(pages, from));
        const size_t at = (size_t)token * a.h_q + head, out_row = (size_t)slot * all_rows + at;
        if (from >= to) {
            if (wave == 0 && rows.r == 0 && real) a.ws_ml[out_row * 2 + 1] = 0.0f;
            continue;
        }
        // ---- this wavefront's quarter
        const int begin = from + (to - from) * wave / 4, count = __builtin_amdgcn_readfirstlane(from + (to - from) * (wave + 1) / 4 - begin);
        auto numbers = [&](int i) __attribute__((always_inline)) { return i + lane < count ? page_of(a.req, b, (begin + i + lane) * kPage) : -1; };
        const int ahead = numbers(0);
        rows.load(a.q + at * D, real, a.scale);
        rows.walk(count, real ? lim : 0, n, a.pages, a.h_kv, kv, ahead, numbers, [&](int i) __attribute__((always_inline)) { return (begin + i) * kPage; });
        const size_t to_row = Meeting<D>::theirs((unsigned long long)out_row);
        four.meet(
            rows, wave, Meeting<D>::theirs((int)real) != 0,
            [&](int d, const v4f &o, float) __attribute__((always_inline)) { *reinterpret_cast<v4f *>(a.ws_o + to_row * D + d) = o; },
            [&](float top, float l) __attribute__((always_inline)) { a.ws_ml[to_row * 2] = top, a.ws_ml[to_row * 2 + 1] = l; });
    }
}

// D / 4 threads per row: its parts, eight on their way at a time.  Rows of nobody stay as they are.
template <int D>
__global__ __launch_bounds__(256) void attn_q4_join_kernel(PartsArgs a) {
    const long all_rows = (long)a.req.tokens * a.h_q, step = (long)gridDim.x * (1024 / D);
    const int d = 4 * (threadIdx.x % (D / 4)), last = token_at(a.req, a.req.batch), slots = a.prefix_parts + a.parts;
    int group0 = 0, group1 = 0;  // tokens of groups
    if (a.prefix_parts) group0 = token_at(a.req, group_end(a, 0)), group1 = token_at(a.req, group_end(a, a.groups));
    for (long row = (long)blockIdx.x * (1024 / D) + threadIdx.x / (D / 4); row < all_rows; row += step) {
        const int token = (int)(row / a.h_q);
        if (token >= last) return;
        const int first = token >= group0 && token < group1 ? 0 : a.prefix_parts;
        float inv;
        const v4f o = joined(a.ws_ml, a.ws_o + d, D, slots - first, [&](int c) __attribute__((always_inline)) { return (size_t)(first + c) * all_rows + row; }, inv);
        *reinterpret_cast<h4 *>(a.out + row * D + d) = rounded(o, inv);
    }
}

constexpr long kMostWgs = 1L << 22;  // (a launch has fewer than 2^32 threads)
template <int D>
hipError_t launch(const PartsArgs &a, hipStream_t st) {
    PartsArgs rest = a;
    if constexpr (D <= 128) {
        if (a.wide) {
            constexpr size_t lds = Wide<D>::kBytes * 2;
            if (const hipError_t e = allow_dynamic_lds<attn_q4_wide_kernel<D>>(lds); e != hipSuccess) return e;
            attn_q4_wide_kernel<D><<<(unsigned)a.prefix_items, 256, lds, st>>>(a);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            rest.items -= a.prefix_items, rest.prefix_items = 0;
        }
    }
    constexpr size_t lds = Place<D>::LDS;
    if (const hipError_t e = allow_dynamic_lds<attn_q4_parts_kernel<D>>(lds); e != hipSuccess) return e;
    attn_q4_parts_kernel<D><<<(unsigned)(rest.items < kMostWgs ? rest.items : kMostWgs), 256, lds, st>>>(rest);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const long joins = ((long)a.req.tokens * a.h_q + 1024 / D - 1) / (1024 / D);
    attn_q4_join_kernel<D><<<(unsigned)(joins < kMostWgs ? joins : kMostWgs), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int D, bool SPREAD, int WAVES>
hipError_t launch_selected(const SelectedArgs &a, hipStream_t st) {
    constexpr size_t lds = Place<D>::LDS * WAVES / 4;
    if (const hipError_t e = allow_dynamic_lds<attn_q4_selected_kernel<D, SPREAD, WAVES>>(lds); e != hipSuccess) return e;
    const unsigned wgs = (unsigned)((a.places + a.share - 1) / a.share);
    attn_q4_selected_kernel<D, SPREAD, WAVES><<<wgs, 64 * WAVES, lds, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || wgs == 1 || a.share % a.count == 0) return e;  // (no unit is cut)
    attn_q4_join_selected_kernel<D, SPREAD><<<wgs - 1, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int D>
hipError_t launch(const SelectedArgs &a, hipStream_t st) {
    if (a.waves == 8) return a.g <= Rows<D, true>::ROWS ? launch_selected<D, true, 8>(a, st) : launch_selected<D, false, 8>(a, st);
    return a.g <= Rows<D, true>::ROWS ? launch_selected<D, true, 4>(a, st) : launch_selected<D, false, 4>(a, st);
}
template <class Args>
hipError_t launch(const Args &a, int d, hipStream_t st) {
    switch (d) {
        case 64: return launch<64>(a, st);
        case 128: return launch<128>(a, st);
        case 256: return launch<256>(a, st);
    }
    return hipErrorInvalidValue;
}

constexpr int kMostParts = 16;
// Rows of partial results per compute unit, beside one part of all rows: with 256 compute units 16 parts of 273 tokens of 32 heads.  (Blocks that fill the card with their rows need 16 kWgs of them, or 128
// kWgs where they are of 128 rows: more only where most of a call's rows are nobody's or in no group.)
constexpr long kKeptRows = 256 * kWgs;
// Rows and common pages of a group times heads and their size per compute unit from which on pages are taken apart for a workgroup.  Both ways' times, us, with 8 KV heads of 128 values: 256 rows
// behind 40000 positions 108 and 117, 60000 163 and 160; 512 rows behind 6000 50 and 63, 16000 90 and 94, 22000 120 and 117, 26000 138 and 131; 1024 rows behind 6000 79 and 91, 20000 203 and 186; with
// 4 heads of 64: 1024 rows behind 20000 72 and 79.  (640 and 768 rows make a few more workgroups than the card has at once, and are slower: behind 20000 147 and 171, 14000 114 and 152.)
constexpr long kWideFrom = 600000;
// Workgroups that share a block's pages: as many as fill the card, each with a page per wavefront at least
int parts_of(long blocks, int pages, int num_cus) {
    const long fill = ((long)kWgs * num_cus + blocks - 1) / (blocks > 0 ? blocks : 1), most = (pages + 3) / 4;
    const long parts = fill < most ? fill : most;
    return (int)(parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts);
}
// Most parts of `rows` rows, whose partial results are kept for every part; rows times this grow with `rows` and `pages`: a workspace for the largest call serves every smaller one
long most_rows(long rows, long pages, int num_cus) {
    const long parts = pages <= 4 ? 1 : (pages + 3) / 4 < kMostParts ? (pages + 3) / 4 : kMostParts, kept = kKeptRows * num_cus + rows;
    return rows * parts < kept ? rows * parts : kept;
}

}  // namespace

// Equal shares of all places for as many workgroups as the card has at once, a page per wavefront at least.  Whole units where that makes the largest share an eighth larger at most: nothing to
// join.  Half as many workgroups of 8 wavefronts have whole units where 4 do not, or have a list of up to 8 pages at once.  (Heads of 128 values, 8 KV heads, us with and without workgroups of 8:
// 30 requests of 32 pages 18.4 and 24.8, 32 of 32 19.4 and 22.6, 32 of 100 46.0 and 50.3; 1 of 8 7.7 and 9.0, but of 16 9.6 and 9.2 and of 32 13.9 and 9.4, if it were not cut.)
SelectedPlan plan_attention_selected_q4(int tokens, int h_q, int h_kv, int d, int count, int num_cus) {
    SelectedPlan p = {};
    const long units = (long)tokens * h_kv * ((h_q / h_kv + 15) / 16), cus = num_cus > 0 ? num_cus : 1;
    p.places = units * count;
    auto shares = [&](int waves, int least) {
        const long wgs = kWgs * cus * 4 / waves, equal = (p.places + wgs - 1) / wgs;
        p.waves = waves, p.share = equal < least ? least : equal;
    };
    auto whole = [&](int waves) {
        shares(waves, count < waves ? count : waves);
        const long units_only = (p.share + count - 1) / count * count;
        const bool fits = units_only <= p.share + p.share / 8;
        p.share = units_only;
        return fits;
    };
    if (!whole(4) && !whole(8)) shares(4, 4);
    p.wgs = (p.places + p.share - 1) / p.share;
    // (what any call of as many places or fewer needs, where its units are cut)
    const long most = kWgs * cus < (p.places + 3) / 4 ? kWgs * cus : (p.places + 3) / 4;
    p.bytes = 256 + (most > 1 ? (size_t)most * 2 * 16 * (d + 2) * sizeof(float) : 0);
    return p;
}

AttnPartsPlan plan_attention_shared_q4(int batch, int tokens, int h_q, int h_kv, int d, int max_tokens, int max_context, int groups, int group_tokens, int longest, int num_cus) {
    AttnPartsPlan p = {};
    const int g = h_q / h_kv;
    const int forced = tuning().attn_wide_rows;
    group_tokens = group_tokens < tokens ? group_tokens : tokens;  // (a limit may be far above what the call holds)
    const long group_rows = (long)group_tokens * g, common = (longest < max_context ? longest : max_context) / kPage;
    p.wide = d <= 128 && (forced > 0 ? group_rows >= forced : group_rows >= 2 * Wide<128>::ROWS && group_rows * common * h_kv * d >= kWideFrom * num_cus);
    const int rows = p.wide ? Wide<128>::ROWS : 16;
    const long by_group = (long)groups * (((long)group_tokens * g + rows - 1) / rows), by_token = ((long)tokens * g + rows - 1) / rows + groups;
    p.prefix_blocks = by_group < by_token ? by_group : by_token;
    p.blocks = max_tokens * g <= 16 ? batch : ((long)tokens * g + 15) / 16 + batch;
    const long all_rows = (long)tokens * h_q, pages = (max_context + kPage - 1) / kPage, most_common = most_rows(all_rows, common, num_cus), most_own = most_rows(all_rows, pages, num_cus);
    auto within = [&](int parts, long most) { return all_rows * parts > most ? (int)(most / all_rows) : parts; };
    p.prefix_parts = within(parts_of(p.prefix_blocks * h_kv, (int)common, num_cus), most_common);
    p.parts = within(parts_of(p.blocks * h_kv, (int)pages, num_cus), most_own);
    p.bytes = 256 + (size_t)(most_common + most_own) * (d + 2) * sizeof(float);
    return p;
}

hipError_t launch_attention_selected_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const void *pages, const int *selected, int count, const SelectedPlan &p, void *workspace,
                                        void *out, hipStream_t st) {
    SelectedArgs a = {};
    a.q = static_cast<const _Float16 *>(q);
    a.out = static_cast<_Float16 *>(out);
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.selected = selected, a.count = count;
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv, a.head_blocks = (a.g + 15) / 16;
    a.share = p.share, a.places = p.places, a.waves = p.waves;
    a.ws_o = static_cast<float *>(workspace);
    a.ws_ml = a.ws_o + (size_t)p.wgs * 2 * 16 * d;
    a.scale = 1.4426950408889634f / sqrtf((float)d);
    return launch(a, d, st);
}

hipError_t launch_attention_shared_q4(const void *q, const Requests &req, int h_q, int h_kv, int d, const void *pages, const int *group_start, const int *prefix, int groups, int group_tokens,
                                      int longest, const AttnPartsPlan &p, void *workspace, void *out, hipStream_t st) {
    PartsArgs a = {};
    a.q = static_cast<const _Float16 *>(q);
    a.out = static_cast<_Float16 *>(out);
    a.pages = static_cast<const char *>(pages);
    a.req = req;
    a.group_start = group_start, a.prefix = prefix, a.groups = groups, a.group_tokens = group_tokens, a.longest = longest;
    a.h_q = h_q, a.h_kv = h_kv, a.g = h_q / h_kv, a.wide = p.wide;
    a.prefix_parts = p.prefix_parts, a.parts = p.parts;
    a.prefix_items = p.prefix_blocks * h_kv * p.prefix_parts;
    a.items = a.prefix_items + p.blocks * h_kv * p.parts;
    a.ws_o = static_cast<float *>(workspace);
    a.ws_ml = a.ws_o + (size_t)(p.prefix_parts + p.parts) * req.tokens * h_q * d;
    a.scale = 1.4426950408889634f / sqrtf((float)d);
    return launch(a, d, st);
}

}  // namespace qfc
