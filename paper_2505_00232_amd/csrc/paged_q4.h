// The paged 4-bit cache and the batch of requests, as the kernels see them (qfc_q4_cache_t, qfc_requests_t).
//
// A page holds 64 positions of every KV head, one block of 80 d bytes per head: first what attention's score product reads, then what its second
// product reads.  Codes are stored as the operands of v_mfma_f32_16x16x32_f16 in KiB tiles (lane l = (m, r), m = l % 16, r = l / 16), so that they go from memory
// through LDS to a lane in one piece:
//   K codes    four tiles t of 16 positions; lane (m, r) holds position 16 (m / 4) + 4 t + m % 4, of every group j of 32 values the octet
//              32 j + 8 r .. + 7 in a dword.  (Row m of a score tile leaves the matrix core in lane m / 4: a lane ends up with 16 consecutive positions.)
//   K step     binary16 [d / 32][64 positions]
//   K offset   binary16 [64 slots][d / 32], slot = 16 t + m of the position
//   V codes    one tile per group of 32 values; lane (m, r) holds the 16 positions 16 r .. + 15 of the values m (low nibbles) and
//              16 + m (high nibbles) of the group, a byte per position
//   V step, V offset   binary16 [d / 32][64 positions] each
// Nibbles and bytes are in the order in which `word & 0x000F000F` and its shifts give neighbours in pairs: a nibble alone in 16 bits is the binary16
// denormal code * 2^-24, exactly, so the codes are matrix operands without a conversion.
#pragma once
#include "qfc_internal.h"

namespace qfc {

constexpr int kPage = QFC_PAGE_POSITIONS;
static_assert(kPage == 64, "the layout below is one of 64 positions");

template <int D>
struct PageLayout {
    static constexpr int G = D / 32;          // groups of 32 values
    static constexpr int W = G < 4 ? G : 4;   // dwords a lane holds of a K tile in one piece
    static constexpr int kCodesK = 0, kStepK = 32 * D, kOffsetK = 36 * D, kCodesV = 40 * D, kStepV = 72 * D, kOffsetV = 76 * D, kBytes = 80 * D;
    __host__ __device__ static int slot(int p) { return 16 * ((p >> 2) & 3) + 4 * (p >> 4) + (p & 3); }
    // dword of octet 32 j + 8 r of position p
    __host__ __device__ static int code_k(int p, int j, int r) {
        const int s = slot(p), lane = 16 * r + (s & 15);
        return kCodesK + (((s >> 4) * (G / W) + j / W) * 64 + lane) * (4 * W) + (j % W) * 4;
    }
    // byte of the values 32 j + m and 32 j + 16 + m of position p: bytes 0, 2, 1, 3 of a dword are four consecutive positions
    __host__ __device__ static int code_v(int p, int j, int m) {
        return kCodesV + (j * 64 + (p >> 4) * 16 + m) * 16 + (p & 12) + (((p & 1) << 1) | ((p >> 1) & 1));
    }
    __host__ __device__ static int step_k(int p, int j) { return kStepK + (j * kPage + p) * 2; }
    __host__ __device__ static int offset_k(int p, int j) { return kOffsetK + (slot(p) * G + j) * 2; }
    __host__ __device__ static int step_v(int p, int j) { return kStepV + (j * kPage + p) * 2; }
    __host__ __device__ static int offset_v(int p, int j) { return kOffsetV + (j * kPage + p) * 2; }
};
// nibble of value e of an octet in its dword: neighbours 16 bits apart
__host__ __device__ inline int nibble(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// A batch of requests on the device.  What the arrays hold is not known to the host: every index taken from them is bounded here.
struct Requests {
    const int *start, *context, *table;
    int batch, tokens, max_tokens, max_context, width, num_pages;
};
struct Span {
    int first, count, positions;  // rows first .. first + count - 1 are the last `count` of `positions` positions (count may be the larger one)
};
__device__ __forceinline__ Span span_of(const Requests &q, int b) {
    Span s;
    s.first = min(max(q.start[b], 0), q.tokens);
    s.count = min(min(max(q.start[b + 1], s.first), q.tokens) - s.first, q.max_tokens);
    s.positions = min(max(q.context[b], 0), q.max_context);
    return s;
}
// page of position p (below max_context) of request b, -1 where it has none
__device__ __forceinline__ int page_of(const Requests &q, int b, int p) {
    const int page = q.table[(size_t)b * q.width + p / kPage];
    return page >= 0 && page < q.num_pages ? page : -1;
}
// Sums that end at the largest int.
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

// Largest over the lanes (m, r) of all r
__device__ __forceinline__ float over_rows(float x) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = fmaxf(__uint_as_float(a.x), __uint_as_float(a.y));
    const u32x2 b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}

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

// Request of a token (batch: of none) and its span, the same in every lane.  What is known of 64 requests is asked for at once: no second look at memory for the one that it is.
__device__ __forceinline__ int request_of_token(const Requests &q, int token, int lane, Span &s) {
    for (int b0 = 0; b0 < q.batch; b0 += 64) {
        const int b = b0 + lane, mine = min(b, q.batch - 1), end = q.start[mine + 1];
        const Span own = span_of(q, mine);
        const int before = (int)__popcll(__ballot(b < q.batch && end <= token));
        if (before < min(64, q.batch - b0)) {
            s = Span{__builtin_amdgcn_readlane(own.first, before), __builtin_amdgcn_readlane(own.count, before), __builtin_amdgcn_readlane(own.positions, before)};
            return b0 + before;
        }
    }
    s = Span{0, 0, 0};
    return q.batch;
}

// Bounds of pages' keys, on the device (qfc_page_bounds_t): codes [page][h_kv][2][d_head], steps [page][h_kv]
struct PageBounds {
    int8_t *codes;
    float *steps;
    int h_kv, d_head;
};

// Pages and how often tables name them, on the device
struct PagePool {
    void *pages;
    int *references;
    int num_pages, page_bytes;
};

}  // namespace qfc
