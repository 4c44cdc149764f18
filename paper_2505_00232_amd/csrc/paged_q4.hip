// Keys and values of a batch of requests: rotated, quantized to 4 bits and appended to a paged cache (layout: paged_q4.h), and read back from it.
//
// Rotation of the pair (x0, x1) by the angle whose cosine and sine the table holds in 32 bits: fp16(x0 c - x1 s), fp16(x1 c + x0 s), the real
// result rounded once.  Quantization of 32 consecutive values of a head:
//   step = fp16((max - min) / 15), offset = fp16(min + 8 step), code = clamp(rne((x - offset) (1 / step)) + 8, 0, 15)
// with every operation rounded to 32 bits; a value is offset + step (code - 8).  Steps and offsets in binary16: what they round off (2^-11 relative) is little against half a
// step of a 4-bit code, and the codes are taken against the rounded ones.
#include "paged_q4.h"

namespace qfc {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint16_t bits16(_Float16 x) { return __builtin_bit_cast(uint16_t, x); }

// Requests of the tokens of a wavefront, PER of them from `first` on: how many requests end at or before a token.  A lane looks at one request at a time.
template <int PER>
__device__ __forceinline__ int request_of(const Requests &q, int first, int mine, int lane) {
    int count[PER] = {};
    for (int b0 = 0; b0 < q.batch; b0 += 64) {
        const int end = b0 + lane < q.batch ? q.start[b0 + lane + 1] : INT32_MAX;
#pragma unroll
        for (int i = 0; i < PER; ++i) count[i] += __popcll(__ballot(end <= first + i));
    }
    int b = count[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) b = mine == i ? count[i] : b;
    return b;
}

// Tiles of tokens are dealt four by four to the XCDs (workgroup i runs on XCD i % 8): a page's lines, of which each tile has a part, then meet in one L2 (4096 tokens appended and read
// 38.6 us, dealt one by one 39.5).
constexpr int kTiles = 4;
__device__ __forceinline__ int tile_of_block(unsigned x) { return (int)((x / (8 * kTiles) * 8 + x % 8) * kTiles + x / 8 % kTiles); }
// Heads one workgroup takes: as few as still fit the card at once, `fit` workgroups per compute unit
int heads_of_workgroup(long tiles, int heads, long fit) {
    const long per = fit > 0 ? tiles * heads / fit : 1;
    return (int)(per < 1 ? 1 : per > heads ? heads : per);
}
unsigned blocks_of_tiles(long tiles) { return (unsigned)((tiles + 8 * kTiles - 1) / (8 * kTiles) * (8 * kTiles)); }

// x0 c + x1 s, rounded to binary16 once: both products with their rounding errors (fma), their sum with its own (Knuth's two-sum); what the last sum
// rounds off decides its lowest bit (rounding to odd), so that the conversion to binary16 rounds the real result.  Without a correction the plain sum stands
// (a zero keeps its sign, an infinite x gives what it gives).
__device__ __forceinline__ _Float16 rotated(float x0, float c, float x1, float s) {
#pragma clang fp contract(off)  // (the two-sum needs its own roundings)
    const float p = x0 * c, q = x1 * s, sum = p + q, of_q = sum - p;
    const float low = ((p - (sum - of_q)) + (q - of_q)) + (fmaf(x0, c, -p) + fmaf(x1, s, -q));
    const float r = sum + low, off = low - (r - sum);
    const int bits = __float_as_int(r), odd = (bits - ((__float_as_int(off) ^ bits) < 0 ? 1 : 0)) | 1;
    return (_Float16)(low < 0.0f || low > 0.0f ? (off != 0.0f ? __int_as_float(odd) : r) : sum);
}

// An octet of them.  x0 c + x1 s with two roundings is off by 2^-24 (|x0 c| + 2 |sum|) at most; where the values that far to both sides of it round to the same binary16,
// that is the result, and only the others (one in some 700) are worked out as above.
__device__ __forceinline__ h8 rotated8(const h8 &x, const h8 &other, const float (&c)[8], const float (&s)[8]) {
    constexpr float off = 1.25f / 8388608.0f;
    h8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float p = (float)x[e] * c[e], sum = fmaf((float)other[e], s[e], p), size = fabsf(p) + fabsf(sum);
        const _Float16 low = (_Float16)fmaf(-off, size, sum), high = (_Float16)fmaf(off, size, sum);
        y[e] = low;
        if (__builtin_expect(__any(bits16(low) != bits16(high)), 0)) y[e] = rotated((float)x[e], c[e], (float)other[e], s[e]);
    }
    return y;
}

// Eight of the 32 values of a group, the others in the three neighbours of this lane's quad: their codes (value e in bits 4 e .. + 3), and the group's step and offset.
__device__ __forceinline__ uint32_t quantize8(const h8 &x, _Float16 &step, _Float16 &offset) {
#pragma clang fp contract(off)
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h4 lo4 = __builtin_elementwise_min(x.lo, x.hi), hi4 = __builtin_elementwise_max(x.lo, x.hi);
    const h2 lo2 = __builtin_elementwise_min(lo4.lo, lo4.hi), hi2 = __builtin_elementwise_max(hi4.lo, hi4.hi);
    float lo = fminf((float)lo2.x, (float)lo2.y), hi = fmaxf((float)hi2.x, (float)hi2.y);
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, off, 64));
        hi = fmaxf(hi, __shfl_xor(hi, off, 64));
    }
    step = (_Float16)((hi - lo) / 15.0f);
    offset = (_Float16)(lo + 8.0f * (float)step);
    const float inv = step > (_Float16)0.0f ? 1.0f / (float)step : 0.0f, zero = (float)offset;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float u = ((float)x[e] - zero) * inv;
        codes |= (uint32_t)(int)fminf(fmaxf(rintf(u) + 8.0f, 0.0f), 15.0f) << (4 * e);
    }
    return codes;
}

struct AppendArgs {
    const _Float16 *qkv;
    _Float16 *q_out;
    char *pages;
    const float2 *table;  // [positions][rot / 2]: cos, sin
    Requests req;
    int h_q, h_kv, rot, interleaved, heads_per_wg;
};

// A workgroup takes 2048 / D consecutive token rows and heads_per_wg heads, one after the other; a thread one octet of a token's head.  The angles stay in its registers from
// head to head, the next head's octets are on their way.  Bound: the latency of arrays, page table, angles and stores one behind the other where tokens are few (64 requests 7 us), memory
// and instructions about alike where they are many: 4096 tokens, 32 heads on 8 of 128 values, 25 us for 89 MB (3.5 TB/s).
template <int D>
__global__ __launch_bounds__(256) void append_q4_kernel(AppendArgs a) {
    typedef PageLayout<D> L;
    constexpr int OCT = D / 8, TT = 256 / OCT, PER = 64 / OCT;
    __shared__ uint32_t vbytes[TT][D / 8];  // values of a token, a byte for every two
    __shared__ int at[TT][2];               // page (-1: none) and position of each token
    const int o = threadIdx.x % OCT, tt = threadIdx.x / OCT, lane = threadIdx.x & 63;
    const int tok0 = tile_of_block(blockIdx.x) * TT, tok = tok0 + tt;
    if (tok0 >= a.req.tokens) return;
    const int heads = a.h_q + 2 * a.h_kv, head0 = (int)blockIdx.y * a.heads_per_wg, head1 = min(head0 + a.heads_per_wg, heads);

    // An octet and what it is rotated with, a head ahead, the first before anything is known of the requests
    const int half = a.rot / 2;
    const bool turns = 8 * o < a.rot, first = 8 * o < half;
    const int partner = !turns || a.interleaved ? o : first ? o + half / 8 : o - half / 8;
    const _Float16 *src = a.qkv + ((size_t)min(tok, a.req.tokens - 1) * heads + head0) * D;
    h8 x_next = *reinterpret_cast<const h8 *>(src + 8 * o), other_next = *reinterpret_cast<const h8 *>(src + 8 * partner);

    const int b = request_of<PER>(a.req, tok0 + tt / PER * PER, tt % PER, lane);
    bool mine = tok < a.req.tokens && b < a.req.batch;
    int pos = -1, page = -1;
    if (mine) {
        const Span s = span_of(a.req, b);
        mine = tok >= s.first && tok - s.first < s.count;
        pos = s.positions - s.count + tok - s.first;
        if (mine && pos >= 0) page = page_of(a.req, b, pos);
    }
    if (o == 0) {
        at[tt][0] = page;
        at[tt][1] = pos;
    }
    // cosine and signed sine of the octet's values
    float c[8], s[8];
    if (turns && mine && head0 < a.h_q + a.h_kv) {
        const float2 *row = a.table + (size_t)max(pos, 0) * half;
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 t = row[4 * o + e / 2];
                c[e] = t.x;
                s[e] = e & 1 ? t.y : -t.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 t = row[(first ? 8 * o : 8 * o - half) + e];
                c[e] = t.x;
                s[e] = first ? -t.y : t.y;
            }
        }
    }
    for (int head = head0; head < head1; ++head) {
        h8 x = x_next;
        const h8 other = a.interleaved ? __builtin_shufflevector(x, x, 1, 0, 3, 2, 5, 4, 7, 6) : other_next;
        src += head + 1 < head1 ? D : 0;
        x_next = *reinterpret_cast<const h8 *>(src + 8 * o);
        other_next = *reinterpret_cast<const h8 *>(src + 8 * partner);
        if (head < a.h_q + a.h_kv && turns && mine) x = rotated8(x, other, c, s);
        if (head < a.h_q) {
            if (mine) *reinterpret_cast<h8 *>(a.q_out + ((size_t)tok * a.h_q + head) * D + 8 * o) = x;
            continue;
        }
        _Float16 step, offset;
        const uint32_t codes = quantize8(x, step, offset);
        const int j = o / 4, in_page = pos & (kPage - 1);
        if (head < a.h_q + a.h_kv) {
            if (page < 0) continue;
            char *dst = a.pages + ((size_t)page * a.h_kv + (head - a.h_q)) * L::kBytes;
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= ((codes >> (4 * e)) & 15u) << nibble(e);
            *reinterpret_cast<uint32_t *>(dst + L::code_k(in_page, j, o & 3)) = w;
            if ((o & 3) == 0) {
                *reinterpret_cast<_Float16 *>(dst + L::step_k(in_page, j)) = step;
                *reinterpret_cast<_Float16 *>(dst + L::offset_k(in_page, j)) = offset;
            }
            continue;
        }
        const int kv = head - a.h_q - a.h_kv;
        // low nibbles are the octets 0 and 1 of a group, high ones 2 and 3: the lane two further has the other half; each packs four bytes
        const uint32_t theirs = __shfl_xor(codes, 2, 64);
        const bool high = (o & 2) != 0;
        const uint32_t lo4 = high ? theirs >> 16 : codes & 0xFFFFu, hi4 = high ? codes >> 16 : theirs & 0xFFFFu;
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w |= (((lo4 >> (4 * e)) & 15u) | (((hi4 >> (4 * e)) & 15u) << 4)) << (8 * e);
        vbytes[tt][4 * j + 2 * (o & 1) + (high ? 1 : 0)] = w;
        if (page >= 0 && (o & 3) == 0) {
            char *dst = a.pages + ((size_t)page * a.h_kv + kv) * L::kBytes;
            *reinterpret_cast<_Float16 *>(dst + L::step_v(in_page, j)) = step;
            *reinterpret_cast<_Float16 *>(dst + L::offset_v(in_page, j)) = offset;
        }
        __syncthreads();
        // a thread: one byte column of four tokens, as one dword where they are four positions of one dword
        const int col = threadIdx.x % (D / 2), t4 = threadIdx.x / (D / 2) * 4;
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const uint8_t *>(vbytes[t4 + i])[col];
        const int page0 = at[t4][0], pos0 = at[t4][1];
        bool whole = page0 >= 0 && (pos0 & 3) == 0;
#pragma unroll
        for (int i = 1; i < 4; ++i) whole = whole && at[t4 + i][0] == page0 && at[t4 + i][1] == pos0 + i;
        if (whole) {
            char *dst = a.pages + ((size_t)page0 * a.h_kv + kv) * L::kBytes + L::code_v(pos0 & (kPage - 1), col / 16, col % 16);
            *reinterpret_cast<uint32_t *>(dst) = v[0] | v[2] << 8 | v[1] << 16 | v[3] << 24;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int pg = at[t4 + i][0];
                if (pg >= 0)
                    a.pages[((size_t)pg * a.h_kv + kv) * L::kBytes + L::code_v(at[t4 + i][1] & (kPage - 1), col / 16, col % 16)] = (char)v[i];
            }
        }
        __syncthreads();
    }
}

struct ReadArgs {
    const char *pages;
    _Float16 *k, *v;  // [tokens, h_kv, D]
    Requests req;
    int h_kv, heads_per_wg;
};

// The values the cache holds for the requests' new tokens; zeros where a token has no page.  Bound: latency, arrays, table, codes and stores one behind the other (64 requests 4 us, 4096
// tokens on 8 heads of 128 values 13 us for 22 MB).
template <int D>
__global__ __launch_bounds__(256) void read_q4_kernel(ReadArgs a) {
    typedef PageLayout<D> L;
    constexpr int OCT = D / 8, TT = 256 / OCT, PER = 64 / OCT;
    const int o = threadIdx.x % OCT, tt = threadIdx.x / OCT, lane = threadIdx.x & 63;
    const int tok0 = tile_of_block(blockIdx.x) * TT, tok = tok0 + tt;
    const int b = request_of<PER>(a.req, tok0 + tt / PER * PER, tt % PER, lane);
    if (tok >= a.req.tokens || b >= a.req.batch) return;
    const Span s = span_of(a.req, b);
    if (tok < s.first || tok - s.first >= s.count) return;
    const int pos = s.positions - s.count + tok - s.first, page = pos >= 0 ? page_of(a.req, b, pos) : -1;
    const int p = pos & (kPage - 1), j = o / 4, kv1 = min(((int)blockIdx.y + 1) * a.heads_per_wg, a.h_kv);
#pragma unroll 2
    for (int kv = (int)blockIdx.y * a.heads_per_wg; kv < kv1; ++kv) {
        h8 k = {}, v = {};
        if (page >= 0) {
            const char *src = a.pages + ((size_t)page * a.h_kv + kv) * L::kBytes;
            const uint32_t w = *reinterpret_cast<const uint32_t *>(src + L::code_k(p, j, o & 3));
            const float sk = (float)*reinterpret_cast<const _Float16 *>(src + L::step_k(p, j)), ok = (float)*reinterpret_cast<const _Float16 *>(src + L::offset_k(p, j));
            const float sv = (float)*reinterpret_cast<const _Float16 *>(src + L::step_v(p, j)), ov = (float)*reinterpret_cast<const _Float16 *>(src + L::offset_v(p, j));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                k[e] = (_Float16)fmaf((float)((w >> nibble(e)) & 15u) - 8.0f, sk, ok);
                const uint32_t byte = (uint8_t)src[L::code_v(p, j, 8 * (o & 1) + e)];
                v[e] = (_Float16)fmaf((float)((o & 2 ? byte >> 4 : byte) & 15u) - 8.0f, sv, ov);
            }
        }
        const size_t dst = ((size_t)tok * a.h_kv + kv) * D + 8 * o;
        *reinterpret_cast<h8 *>(a.k + dst) = k;
        *reinterpret_cast<h8 *>(a.v + dst) = v;
    }
}

// table[p][i] = amplitude (cos, sin) of p f_i, in fp64 as far as the rounding to 32 bits; the angles from `first` on
__global__ __launch_bounds__(256) void rotary_table_kernel(long first, int half, int positions, double log_base, double factor, double turns, double low, double high, double amplitude,
                                                           float2 *__restrict__ table) {
    const long idx = first + (long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (long)positions * half) return;
    const int i = (int)(idx % half), pos = (int)(idx / half);
    double f = exp(-(double)i / (double)half * log_base);
    // a wave that turns often within `turns` 2 pi positions keeps its frequency, one that hardly turns has it divided
    const double keep = turns > 0.0 ? fmin(fmax((turns * f - low) / (high - low), 0.0), 1.0) : 0.0;
    f = keep * f + (1.0 - keep) * f / factor;
    double sn, cs;
    sincos((double)pos * f, &sn, &cs);
    table[idx] = make_float2((float)(amplitude * cs), (float)(amplitude * sn));
}

}  // namespace

hipError_t launch_rotary_table(int rot, double base, double factor, int original, double low, double high, double amplitude, int positions, float *table, hipStream_t st) {
    const long total = (long)positions * (rot / 2), most = 1L << 28;  // (a launch has fewer than 2^32 threads)
    for (long first = 0; first < total; first += most)
        rotary_table_kernel<<<(unsigned)(((total - first < most ? total - first : most) + 255) / 256), 256, 0, st>>>(
            first, rot / 2, positions, log(base), factor, (double)original / (2.0 * M_PI), low, high, amplitude, reinterpret_cast<float2 *>(table));
    return hipGetLastError();
}

hipError_t launch_append_q4(const void *qkv, const Requests &req, int h_q, int h_kv, int d, int rot, bool interleaved, const float *table, void *pages, void *q_out,
                            int num_cus, hipStream_t st) {
    AppendArgs a;
    a.qkv = static_cast<const _Float16 *>(qkv);
    a.q_out = static_cast<_Float16 *>(q_out);
    a.pages = static_cast<char *>(pages);
    a.table = reinterpret_cast<const float2 *>(table);
    a.req = req;
    a.h_q = h_q, a.h_kv = h_kv, a.rot = rot, a.interleaved = interleaved;
    const int tt = 2048 / d, heads = h_q + 2 * h_kv;
    const long tiles = (req.tokens + tt - 1) / tt;
    // (70 registers: seven fit.  4096 tokens, 32 heads on 8 of 128 values, with 4 / 5 / 6 / 7 / 8 of them: 28 / 25 / 25 / 30 / 30 us)
    a.heads_per_wg = heads_of_workgroup(tiles, heads, 6L * num_cus);
    const dim3 grid(blocks_of_tiles(tiles), (unsigned)((heads + a.heads_per_wg - 1) / a.heads_per_wg));
    if (d == 64)
        append_q4_kernel<64><<<grid, 256, 0, st>>>(a);
    else if (d == 128)
        append_q4_kernel<128><<<grid, 256, 0, st>>>(a);
    else
        append_q4_kernel<256><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_read_q4(const Requests &req, int h_kv, int d, const void *pages, void *k, void *v, int num_cus, hipStream_t st) {
    ReadArgs a;
    a.pages = static_cast<const char *>(pages);
    a.k = static_cast<_Float16 *>(k);
    a.v = static_cast<_Float16 *>(v);
    a.req = req;
    const int tt = 2048 / d;
    const long tiles = (req.tokens + tt - 1) / tt;
    a.h_kv = h_kv, a.heads_per_wg = heads_of_workgroup(tiles, h_kv, 8L * num_cus);
    const dim3 grid(blocks_of_tiles(tiles), (unsigned)((h_kv + a.heads_per_wg - 1) / a.heads_per_wg));
    if (d == 64)
        read_q4_kernel<64><<<grid, 256, 0, st>>>(a);
    else if (d == 128)
        read_q4_kernel<128><<<grid, 256, 0, st>>>(a);
    else
        read_q4_kernel<256><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace qfc
