// The pages of a cache as things that requests take, share, let go and are moved between: references[page] table entries name a page, none: it is free.
//
// Free pages are given lowest first and to entries in order, so that the result is the same whatever the order in which wavefronts run: the i-th entry that lacks a page gets the i-th free
// page.  A first launch writes the free pages as a bit each, their number in every 1024 (a chunk), and how many pages each row lacks; in the last one a wavefront per row adds
// up what the rows before its own lack (many rows: sums of runs, from a launch between the two), finds the chunk its first page is in, and takes bits one after the other.  The bits are a copy: what
// other wavefronts enter into references meanwhile changes nothing here.
#include "paged_q4.h"

namespace qfc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 1024, kWords = kChunk / 64;
// Rows from which on what they lack is added up in runs, by a launch of its own.  One entry per row, us with and without: take of 2048 rows 25.2 and 21.7, of 4096 28.4 and 30.0, of 131072 208 and
// 1820 (without, every row reads those of all before it); fork of 4096 rows 44.6 and 42.5, of 8192 63.5 and 78.0, of 131072 687 and 6860.
constexpr int kRun = 1024, kManyRows = 4096;

struct PagesArgs {
    char *pages;
    int *references;
    int num_pages, page_bytes;
    int *table;          // [batch, width]: the rows that get pages
    const int *positions;
    int batch, width;
    const int *from, *parents;  // [from_batch, from_width], [batch]: forks
    int from_batch, from_width;
    int *missing;        // or null
    uint64_t *bits;      // of free pages
    int *free_of, *need, *need_of;  // [chunks], [batch], [batch / kRun]
    int *source, *target, *before;  // compaction: moves, free pages before each chunk
    int chunks, slices;
    PageBounds bounds;  // of the pages, moved with them (codes null: none)
};

__device__ __forceinline__ bool is_page(int page, int num_pages) { return page >= 0 && page < num_pages; }
__device__ __forceinline__ int pages_for(int positions, int width) {
    const int most = width > INT32_MAX / kPage ? INT32_MAX : width * kPage;
    return (int)(((long)min(max(positions, 0), most) + kPage - 1) / kPage);
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}
__device__ __forceinline__ int sum_of(const int *x, int count, int lane) {
    int s = 0;
    for (int i = lane; i < count; i += 64) s += x[i];
    return wave_sum(s);
}

// The part-filled page of a child: its entry, and the page of its parent (-1: there is none to copy)
struct Part {
    int entry, page;
};
__device__ __forceinline__ Part part_of(const PagesArgs &a, int b) {
    const int parent = a.parents[b], n = min(max(a.positions[b], 0), a.from_width > INT32_MAX / kPage ? INT32_MAX : a.from_width * kPage);
    const Part none = {-1, -1};
    if (parent < 0 || parent >= a.from_batch || n % kPage == 0 || n / kPage >= a.width) return none;
    const int page = a.from[(size_t)parent * a.from_width + n / kPage];
    return Part{n / kPage, is_page(page, a.num_pages) ? page : -1};
}

// ---- first launch: free pages (workgroups up to chunks / 4), what rows lack (the others, a wavefront per row)
enum { kTake = 0, kFork = 1, kCompact = 2 };
__device__ __forceinline__ void count_chunk(const PagesArgs &a, int chunk, int lane) {
    const long first = (long)chunk * kChunk;
    int held[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) held[i] = a.references[min(first + 64 * i + lane, (long)a.num_pages - 1)];
    uint64_t mine = 0;
    int count = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const uint64_t word = __ballot(held[i] <= 0 && first + 64 * i + lane < a.num_pages);
        count += __popcll(word);
        mine = lane == i ? word : mine;
    }
    if (lane < kWords) a.bits[(size_t)chunk * kWords + lane] = mine;
    if (lane == 0) a.free_of[chunk] = count;
}
template <int KIND>
__device__ __forceinline__ void count_row(const PagesArgs &a, int b, int lane) {
    int lacks = 0;
    if constexpr (KIND == kFork) {
        lacks = part_of(a, b).page >= 0;
    } else {
        const int entries = pages_for(a.positions[b], a.width);
        for (int e = lane; e < entries; e += 64) lacks += !is_page(a.table[(size_t)b * a.width + e], a.num_pages);
        lacks = wave_sum(lacks);
    }
    if (lane == 0) a.need[b] = lacks;
}
template <int KIND>
__global__ __launch_bounds__(256) void count_pages_kernel(PagesArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), counting = (a.chunks + 3) / 4;
    if ((int)blockIdx.x < counting) {
        const int chunk = (int)blockIdx.x * 4 + wave;
        if (chunk < a.chunks) count_chunk(a, chunk, lane);
    } else if constexpr (KIND != kCompact) {
        const int b = ((int)blockIdx.x - counting) * 4 + wave;
        if (b < a.batch) count_row<KIND>(a, b, lane);
    }
}

// What the rows of each whole run lack
__global__ __launch_bounds__(256) void sum_rows_kernel(PagesArgs a) {
    const int lane = threadIdx.x & 63, run = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (run >= a.batch / kRun) return;
    const int sum = sum_of(a.need + (size_t)run * kRun, kRun, lane);
    if (lane == 0) a.need_of[run] = sum;
}
// What the rows before b lack
__device__ __forceinline__ int lacking_before(const PagesArgs &a, int b, int lane) {
    if (a.batch <= kManyRows) return sum_of(a.need, b, lane);
    return sum_of(a.need_of, b / kRun, lane) + sum_of(a.need + b / kRun * kRun, b % kRun, lane);
}

// The free pages from the rank-th on, in ascending order, up to 64 at a time
struct FreePages {
    const PagesArgs &a;
    const int lane;
    int chunk, word;
    uint64_t held, bits;  // lane i: word i of the chunk; what is left of the present word
    __device__ __forceinline__ FreePages(const PagesArgs &args, int l, int rank) : a(args), lane(l), chunk(0), word(0), held(0), bits(0) {
        bool found = false;
        for (; chunk < a.chunks; chunk += 64) {
            int upto = chunk + lane < a.chunks ? a.free_of[chunk + lane] : 0;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int other = __shfl_up(upto, off, 64);
                upto += lane >= off ? other : 0;
            }
            const uint64_t past = __ballot(upto > rank);
            if (past) {
                const int l0 = __ffsll((unsigned long long)past) - 1;
                rank -= l0 ? __shfl(upto, l0 - 1, 64) : 0;
                chunk += l0;
                found = true;
                break;
            }
            rank -= __shfl(upto, 63, 64);
        }
        if (!found) {
            chunk = a.chunks;
            return;
        }
        fetch();
        while (word < kWords - 1 && __popcll(bits) <= rank) {
            rank -= __popcll(bits);
            bits = at(++word);
        }
        for (; rank > 0 && bits; --rank) bits &= bits - 1;
    }
    __device__ __forceinline__ uint64_t at(int w) const { return __shfl((unsigned long long)held, w, 64); }
    __device__ __forceinline__ void fetch() {
        held = lane < kWords ? a.bits[(size_t)chunk * kWords + lane] : 0;
        word = 0;
        bits = at(0);
    }
    // lane i: the i-th of the next `count` (up to 64; -1: there are no more); `buffer`: 64 ints of the wavefront
    __device__ __forceinline__ int next(int count, volatile int *buffer) {
        int got = 0, mine = -1;
        while (got < count && chunk < a.chunks) {
            if (!bits) {
                if (word < kWords - 1)
                    bits = at(++word);
                else if (++chunk < a.chunks)
                    fetch();
                continue;
            }
            const int here = min(__popcll(bits), count - got), rank = __popcll(bits & ((1ull << lane) - 1));
            const bool taken = (bits >> lane & 1) && rank < here;
            if (taken) buffer[rank] = chunk * kChunk + word * 64 + lane;
            __builtin_amdgcn_wave_barrier();
            if (lane >= got && lane < got + here) mine = buffer[lane - got];
            __builtin_amdgcn_wave_barrier();
            bits &= ~__ballot(taken);
            got += here;
        }
        return mine;
    }
};

__device__ __forceinline__ void say_missing(const PagesArgs &a, int needed, int lane) {
    if (!a.missing) return;
    const int there = sum_of(a.free_of, a.chunks, lane);
    if (lane == 0) *a.missing = max(needed - there, 0);
}

// Pages for the entries of row b that lack one, by a wavefront
__device__ __forceinline__ void take_row(const PagesArgs &a, int b, int lane, int *buffer) {
    const int need = a.need[b], before = lacking_before(a, b, lane);
    if (b == a.batch - 1) say_missing(a, before + need, lane);
    if (need == 0) return;
    FreePages free_pages(a, lane, before);
    const int entries = pages_for(a.positions[b], a.width);
    int *row = a.table + (size_t)b * a.width;
    for (int e0 = 0; e0 < entries; e0 += 64) {
        const int e = e0 + lane;
        const bool lacks = e < entries && !is_page(row[e], a.num_pages);
        const uint64_t all = __ballot(lacks);
        if (!all) continue;
        const int page = __shfl(free_pages.next(__popcll(all), buffer), __popcll(all & ((1ull << lane) - 1)), 64);
        if (lacks) {
            row[e] = page;
            if (page >= 0) a.references[page] = 1;
        }
    }
}
// Bound: latency (counts, chunk, bits, one after the other)
__global__ __launch_bounds__(256) void take_pages_kernel(PagesArgs a) {
    __shared__ int buffers[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = (int)blockIdx.x * 4 + wave;
    if (b < a.batch) take_row(a, b, lane, buffers[wave]);
}
// Small pools and few rows: both steps in one launch, by one workgroup.  (A launch costs the host 2.7 us; with more rows the 16 wavefronts take longer than that one after the other.)
constexpr int kSmallPool = 16 * kChunk, kFewRows = 64;
__global__ __launch_bounds__(1024) void take_few_pages_kernel(PagesArgs a) {
    __shared__ int buffers[16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (wave < a.chunks) count_chunk(a, wave, lane);
    for (int b = wave; b < a.batch; b += 16) count_row<kTake>(a, b, lane);
    __syncthreads();  // (what the workgroup has written to memory is seen by all of it)
    for (int b = wave; b < a.batch; b += 16) take_row(a, b, lane, buffers[wave]);
}

// Copies bytes [from, to) of a page, by the threads of a workgroup; both multiples of 16.  Four of a thread's loads on their way at once.  (A page may end just below 2^31 bytes: what is added to places
// in it passes 32 bits.)
__device__ __forceinline__ void copy_bytes(char *dst, const char *src, int from, int to) {
    for (unsigned at = (unsigned)from + threadIdx.x * 16; at < (unsigned)to; at += 4 * 4096) {
        u32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4 *>(src + min(at + 4096 * i, (unsigned)to - 16));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + 4096 * i < (unsigned)to) *reinterpret_cast<u32x4 *>(dst + at + 4096 * i) = x[i];
    }
}
// Bounds of a page's keys go where the page goes
__device__ __forceinline__ void copy_bounds(const PageBounds &to, int target, const PageBounds &from, int source) {
    if (!from.codes) return;
    const size_t bytes = (size_t)from.h_kv * 2 * from.d_head;
    for (size_t i = (size_t)threadIdx.x * 16; i < bytes; i += 4096) *reinterpret_cast<u32x4 *>(to.codes + target * bytes + i) = *reinterpret_cast<const u32x4 *>(from.codes + source * bytes + i);
    for (int i = threadIdx.x; i < from.h_kv; i += 256) to.steps[(size_t)target * from.h_kv + i] = from.steps[(size_t)source * from.h_kv + i];
}
__device__ __forceinline__ int slice_at(const PagesArgs &a, int slice) { return (int)((long)a.page_bytes / 16 * slice / a.slices) * 16; }

// Row b of the children: whole pages are its parent's, counted once more; the page in part filled is copied, a slice of it by each of the row's workgroups.
__global__ __launch_bounds__(256) void fork_pages_kernel(PagesArgs a) {
    __shared__ int buffers[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = (int)(blockIdx.x / a.slices), slice = (int)(blockIdx.x % a.slices);
    const Part part = part_of(a, b);
    int fresh = -1;
    const bool last = b == a.batch - 1 && slice == 0 && wave == 0;
    if (part.page >= 0 || (last && a.missing)) {
        const int before = lacking_before(a, b, lane);
        if (last) say_missing(a, before + (part.page >= 0), lane);
        if (part.page >= 0) {
            FreePages free_pages(a, lane, before);
            fresh = __shfl(free_pages.next(1, buffers[wave]), 0, 64);
        }
    }
    if (slice == 0) {
        const int parent = a.parents[b];
        const bool known = parent >= 0 && parent < a.from_batch;
        const int whole = known ? min(max(a.positions[b], 0) / kPage, a.from_width) : 0;
        for (int e = threadIdx.x; e < a.width; e += 256) {
            int page = e < whole ? a.from[(size_t)parent * a.from_width + e] : -1;
            page = is_page(page, a.num_pages) ? page : -1;
            if (page >= 0) atomicAdd(a.references + page, 1);
            a.table[(size_t)b * a.width + e] = e == part.entry ? fresh : page;
        }
        if (threadIdx.x == 0 && fresh >= 0) a.references[fresh] = 1;
        if (fresh >= 0) copy_bounds(a.bounds, fresh, a.bounds, part.page);
    }
    if (fresh >= 0) copy_bytes(a.pages + (size_t)fresh * a.page_bytes, a.pages + (size_t)part.page * a.page_bytes, slice_at(a, slice), slice_at(a, slice + 1));
}

// Entries from ceil(keep / 64) on are dropped
__global__ __launch_bounds__(256) void free_pages_kernel(int *references, int num_pages, int *table, const int *keep, int batch, int width) {
    const long all = (long)batch * width, step = (long)gridDim.x * 256;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int b = (int)(i / width), e = (int)(i % width);
        if (keep && e < pages_for(keep[b], width)) continue;
        const int page = table[i];
        if (is_page(page, num_pages)) atomicSub(references + page, 1);
        table[i] = -1;
    }
}

// Pairs of pages, a slice of one per workgroup, one after the other.  Bound: memory (3000 pages of 80 KiB 101 us: 4.9 TB/s, a plain copy 5.06).
__global__ __launch_bounds__(256) void copy_pages_kernel(const char *from, int from_pages, char *to, int to_pages, const int *source, const int *target, int count, int page_bytes, int slices,
                                                         PageBounds from_bounds, PageBounds to_bounds) {
    const long all = (long)count * slices;
    for (long i = blockIdx.x; i < all; i += gridDim.x) {
        const int pair = (int)(i / slices), slice = (int)(i % slices), s = source[pair], t = target[pair];
        if (!is_page(s, from_pages) || !is_page(t, to_pages)) continue;
        if (slice == 0) copy_bounds(to_bounds, t, from_bounds, s);
        copy_bytes(to + (size_t)t * page_bytes, from + (size_t)s * page_bytes, (int)((long)page_bytes / 16 * slice / slices) * 16, (int)((long)page_bytes / 16 * (slice + 1) / slices) * 16);
    }
}

// ---- compaction.  U pages are in use: the i-th of those with numbers from U on goes to the i-th free page below U.  A wavefront per chunk lists both.
__device__ __forceinline__ void list_chunk(const PagesArgs &a, int chunk, int lane, int *used_out) {
    const uint64_t held = lane < kWords ? a.bits[(size_t)chunk * kWords + lane] : 0;  // lane w: word w
    int before = sum_of(a.free_of, chunk, lane);
    const int free_all = before + sum_of(a.free_of + chunk, a.chunks - chunk, lane), used = a.num_pages - free_all;
    // free pages below U, and with them the used ones: U lies in chunk cut
    const int cut = used / kChunk, left = used - cut * kChunk - 64 * lane;
    const uint64_t at_cut = cut < a.chunks && lane < kWords && left > 0 ? a.bits[(size_t)cut * kWords + lane] & (left >= 64 ? ~0ull : (1ull << left) - 1) : 0;
    const int free_below = (cut >= chunk ? before + sum_of(a.free_of + chunk, min(cut, a.chunks) - chunk, lane) : sum_of(a.free_of, cut, lane)) + wave_sum((int)__popcll(at_cut));
    if (lane == 0) {
        a.before[chunk] = before;
        if (chunk == 0) {
            a.before[a.chunks] = used;
            a.before[a.chunks + 1] = free_below;
            if (used_out) *used_out = used;
        }
    }
    const int used_below = used - free_below;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const uint64_t word = __shfl((unsigned long long)held, w, 64);
        const long page = (long)chunk * kChunk + 64 * w + lane;
        const int free_before = before + (int)__popcll(word & ((1ull << lane) - 1));
        if (page < a.num_pages) {
            const bool is_free = word >> lane & 1;
            if (is_free && page < used) a.target[free_before] = (int)page;
            if (!is_free && page >= used) a.source[(int)page - free_before - used_below] = (int)page;
        }
        before += (int)__popcll(word);
    }
}
__global__ __launch_bounds__(256) void list_moves_kernel(PagesArgs a, int *used_out) {
    const int chunk = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (chunk < a.chunks) list_chunk(a, chunk, threadIdx.x & 63, used_out);
}
// Small pools: counted and listed in one launch, by one workgroup (5000 pages 5.6 us, two launches 2.4 and 5.2)
__global__ __launch_bounds__(1024) void list_few_moves_kernel(PagesArgs a, int *used_out) {
    const int chunk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (chunk < a.chunks) count_chunk(a, chunk, lane);
    __syncthreads();  // (what the workgroup has written to memory is seen by all of it)
    if (chunk < a.chunks) list_chunk(a, chunk, lane, used_out);
}

// Moves (a slice of a page per workgroup, one after the other) and tables (the other workgroups)
__global__ __launch_bounds__(256) void move_pages_kernel(PagesArgs a, int movers) {
    const int used = a.before[a.chunks], moves = a.before[a.chunks + 1];  // (as many free pages below U as used ones from there on)
    if ((int)blockIdx.x < movers) {
        for (long i = blockIdx.x; i < (long)moves * a.slices; i += movers) {
            const int k = (int)(i / a.slices), slice = (int)(i % a.slices), s = a.source[k], t = a.target[k];
            if (slice == 0 && threadIdx.x == 0) {
                a.references[t] = a.references[s];
                a.references[s] = 0;
            }
            if (slice == 0) copy_bounds(a.bounds, t, a.bounds, s);
            copy_bytes(a.pages + (size_t)t * a.page_bytes, a.pages + (size_t)s * a.page_bytes, slice_at(a, slice), slice_at(a, slice + 1));
        }
        return;
    }
    const long all = (long)a.batch * a.width, step = (long)(gridDim.x - movers) * 256;
    for (long i = (long)(blockIdx.x - movers) * 256 + threadIdx.x; i < all; i += step) {
        const int page = a.table[i];
        if (!is_page(page, a.num_pages) || page < used) continue;
        const int chunk = page / kChunk, w = page % kChunk / 64;
        int free_before = a.before[chunk];
        for (int j = 0; j < w; ++j) free_before += __popcll(a.bits[(size_t)chunk * kWords + j]);
        const uint64_t word = a.bits[(size_t)chunk * kWords + w];
        free_before += __popcll(word & ((1ull << (page % 64)) - 1));
        if (!(word >> (page % 64) & 1)) a.table[i] = a.target[page - free_before - (used - moves)];  // (an entry that names a free page stays)
    }
}

PagesArgs args_of(const PagePool &pool, void *workspace, int batch) {
    PagesArgs a = {};
    a.pages = static_cast<char *>(pool.pages);
    a.references = pool.references, a.num_pages = pool.num_pages, a.page_bytes = pool.page_bytes;
    a.chunks = (int)(((long)pool.num_pages + kChunk - 1) / kChunk), a.batch = batch;
    char *at = static_cast<char *>(workspace);
    auto part = [&](size_t bytes) {
        char *p = at;
        at += (bytes + 15) / 16 * 16;
        return p;
    };
    a.bits = reinterpret_cast<uint64_t *>(part((size_t)a.chunks * kWords * 8));
    a.free_of = reinterpret_cast<int *>(part((size_t)a.chunks * 4));
    a.need = reinterpret_cast<int *>(part((size_t)batch * 4));
    a.need_of = reinterpret_cast<int *>(part((size_t)(batch / kRun) * 4));
    a.before = reinterpret_cast<int *>(part((size_t)(a.chunks + 2) * 4));
    a.source = reinterpret_cast<int *>(part((size_t)(pool.num_pages / 2 + 1) * 4));
    a.target = reinterpret_cast<int *>(part((size_t)(pool.num_pages / 2 + 1) * 4));
    return a;
}
unsigned fours(long x) { return (unsigned)((x + 3) / 4); }
void sum_rows(const PagesArgs &a, hipStream_t st) {
    if (a.batch > kManyRows) sum_rows_kernel<<<fours(a.batch / kRun), 256, 0, st>>>(a);
}
// Workgroups per page: 16 KiB each where pages are many, as many as fill the card where they are few
int slices_of(int page_bytes, long pages, int num_cus) {
    const long most = page_bytes / 4096 > 1 ? page_bytes / 4096 : 1, least = (page_bytes + 16383L) / 16384, fill = (2L * num_cus + pages - 1) / (pages > 0 ? pages : 1);
    return (int)(fill < least ? least : fill > most ? most : fill);
}

}  // namespace

size_t pages_workspace(int num_pages, int batch) {
    const size_t chunks = ((size_t)num_pages + kChunk - 1) / kChunk;
    return 256 + chunks * kWords * 8 + chunks * 8 + (size_t)batch * 4 + (size_t)(batch / kRun) * 4 + 2 * ((size_t)num_pages / 2 + 1) * 4 + 7 * 16;
}

hipError_t launch_copy_pages(const void *from, int from_pages, void *to, int to_pages, int page_bytes, const int *source, const int *target, int count, const PageBounds &from_bounds, const PageBounds &to_bounds,
                             int num_cus, hipStream_t st) {
    const int slices = slices_of(page_bytes, count, num_cus);
    const long all = (long)count * slices, most = 32L * num_cus;
    copy_pages_kernel<<<(unsigned)(all < most ? all : most), 256, 0, st>>>(static_cast<const char *>(from), from_pages, static_cast<char *>(to), to_pages, source, target, count, page_bytes, slices, from_bounds, to_bounds);
    return hipGetLastError();
}

hipError_t launch_take_pages(const PagePool &pool, int *table, const int *positions, int batch, int width, int *missing, void *workspace, hipStream_t st) {
    PagesArgs a = args_of(pool, workspace, batch);
    a.table = table, a.positions = positions, a.width = width, a.missing = missing;
    if (pool.num_pages <= kSmallPool && batch <= kFewRows) {
        take_few_pages_kernel<<<1, 1024, 0, st>>>(a);
        return hipGetLastError();
    }
    count_pages_kernel<kTake><<<fours(a.chunks) + fours(batch), 256, 0, st>>>(a);
    sum_rows(a, st);
    take_pages_kernel<<<fours(batch), 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_fork_pages(const PagePool &pool, const int *from, int from_batch, int from_width, const int *parents, const int *positions, int *table, int batch, int width, int *missing,
                             const PageBounds &bounds, void *workspace, int num_cus, hipStream_t st) {
    PagesArgs a = args_of(pool, workspace, batch);
    a.bounds = bounds;
    a.from = from, a.from_batch = from_batch, a.from_width = from_width, a.parents = parents;
    a.table = table, a.positions = positions, a.width = width, a.missing = missing;
    a.slices = slices_of(a.page_bytes, batch, num_cus);
    while ((long)batch * a.slices > 1L << 23) a.slices = (a.slices + 1) / 2;  // (a launch has fewer than 2^32 threads; batch is below 2^23)
    count_pages_kernel<kFork><<<fours(a.chunks) + fours(batch), 256, 0, st>>>(a);
    sum_rows(a, st);
    fork_pages_kernel<<<(unsigned)batch * a.slices, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_free_pages(int *references, int num_pages, int *table, const int *keep, int batch, int width, int num_cus, hipStream_t st) {
    const long all = ((long)batch * width + 255) / 256, most = 32L * num_cus;
    free_pages_kernel<<<(unsigned)(all < most ? all : most), 256, 0, st>>>(references, num_pages, table, keep, batch, width);
    return hipGetLastError();
}

hipError_t launch_compact_pages(const PagePool &pool, int *table, int batch, int width, int *used, const PageBounds &bounds, void *workspace, int num_cus, hipStream_t st) {
    PagesArgs a = args_of(pool, workspace, batch);
    a.bounds = bounds;
    a.table = table, a.width = width;
    a.slices = slices_of(a.page_bytes, pool.num_pages / 4, num_cus);
    if (pool.num_pages <= kSmallPool) {
        list_few_moves_kernel<<<1, 1024, 0, st>>>(a, used);
    } else {
        count_pages_kernel<kCompact><<<fours(a.chunks), 256, 0, st>>>(a);
        list_moves_kernel<<<fours(a.chunks), 256, 0, st>>>(a, used);
    }
    const long all = ((long)batch * width + 255) / 256, tables = all < 4L * num_cus ? all : 4L * num_cus;
    const long moves = (long)(pool.num_pages / 2 > 0 ? pool.num_pages / 2 : 1) * a.slices, movers = moves < 16L * num_cus ? moves : 16L * num_cus;
    move_pages_kernel<<<(unsigned)(movers + tables), 256, 0, st>>>(a, (int)movers);
    return hipGetLastError();
}

}  // namespace qfc
