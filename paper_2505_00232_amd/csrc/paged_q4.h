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

}  // namespace qfc
