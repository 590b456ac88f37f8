// The pages of the cache: releasing them, giving a sequence the text of another one (a fork), reserving pages for tokens to come, and moving
// the pages that are held to the lowest numbers.
//
// refs[page] counts the block tables' entries (and the caller's own holds) on a page; 0 means that it is free.  Free pages are taken in
// ascending order, by sequences in ascending order and by a sequence's positions in ascending order, so that every call has one result: what is taken
// is known from ranks and not from who comes first.
//
//   index   a bit per page that is held, the number of such pages in front of every 64 (within 4096) and in every 4096
//   select  the r-th free (or held) page by these counts: a search over the 4096s, one over their 64s and one over a word's bits, a wavefront each
//
// The first launch of a call writes the index and how many pages every sequence needs, from what the state is before the call; the second one
// takes them.  Pages that a call releases are free for the next call.  What has to move is pages, at the rate of a copy.  28 layers of 4 KV heads:
// forks of 8 prompts to 15 responses each, 200 MB, 40 us behind an index of 3 to 6 (5.0 TB/s; a copy of 4 GiB runs at 4.9); a compaction that moves
// 640 MB, read and written, 262 us behind a map of 8 (4.95 TB/s).  Small pools are bound by their launches, 3 to 5 us each.  A page each for 128
// sequences in a pool of 16384 pages 7 us, of 75000, with the launch for the index, 11; a compaction in which nothing moves 12 and 13.
#include <algorithm>

#include "hs_internal.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int WORD = 64, CHUNK = 64 * WORD;      // pages of a word of the index, of a chunk

struct page_args {
    int32_t *refs, *table;
    u64* bits;                        // [words] bit i: page 64 w + i is held
    uint32_t *before, *chunk, *need;  // [words] held pages of the chunk in front of the word; [chunks] held pages; [batch] pages wanted
    int n_blocks, max_blocks, batch, words, chunks, extra;
    // sequences
    int32_t *seq_len, *tail, *tail_len, *k_state, *budget_left, *tokens;
    int w_max, tokens_stride;
    const int32_t *parent, *from, *to;
    // the cache: `block` bytes of K and as many of V per page and layer
    char *k, *v;
    unsigned block;
    int layers, max_rows;
    // compaction
    int32_t *moved, *n_live, *pairs, *n_moves;
    uint32_t* err;
};

__device__ __forceinline__ bool is_page(const page_args& a, int p) { return (unsigned)p < (unsigned)a.n_blocks; }
__device__ __forceinline__ void report(const page_args& a, uint32_t bit) { atomicOr(a.err, bit); }
// Pages that a chunk or a word has at all: the last ones may be cut.
__device__ __forceinline__ int pages_in(const page_args& a, int first, int most) { return min(max(a.n_blocks - first, 0), most); }
__device__ __forceinline__ u64 low_bits(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1ull; }
template <bool FREE>
__device__ __forceinline__ u64 marked(const page_args& a, int w) {
    const u64 held = a.bits[w];
    return FREE ? ~held & low_bits(pages_in(a, w * WORD, WORD)) : held;
}
template <bool FREE>
__device__ __forceinline__ int marked_before(const page_args& a, int w) {      // within the chunk
    return FREE ? (w & 63) * WORD - (int)a.before[w] : (int)a.before[w];
}
template <bool FREE>
__device__ __forceinline__ int marked_in_chunk(const page_args& a, int c) {
    if (c >= a.chunks) return 0;
    return FREE ? pages_in(a, c * CHUNK, CHUNK) - (int)a.chunk[c] : (int)a.chunk[c];
}
__device__ __forceinline__ int wave_prefix(int v, int lane) {      // over the lanes up to and including this one
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// Where the r-th marked page is: its chunk, or -1, and its rank there.  By a whole wavefront; r is the same in all lanes.
template <bool FREE>
__device__ __forceinline__ int find_chunk(const page_args& a, int& r, int lane) {
    for (int c0 = 0; c0 < a.chunks; c0 += 64) {
        const int n = marked_in_chunk<FREE>(a, c0 + lane), upto = wave_prefix(n, lane);
        const u64 hit = __ballot(upto > r);
        if (hit) {
            const int at = __ffsll((long long)hit) - 1;
            r -= __shfl(upto - n, at);
            return c0 + at;
        }
        r -= __shfl(upto, 63);
    }
    return -1;
}
template <bool FREE>
__device__ __forceinline__ int select_page(const page_args& a, int r, int lane) {
    const int c = find_chunk<FREE>(a, r, lane);
    if (c < 0) return -1;
    const int w = c * 64 + lane;
    const bool there = w < a.words;
    const int first = there ? marked_before<FREE>(a, w) : INT32_MAX;
    const u64 mine = there ? marked<FREE>(a, w) : 0ull;
    const int at = 63 - __clzll((long long)__ballot(first <= r));
    const int k = r - __shfl(first, at);
    const u64 word = ((u64)(unsigned)__shfl((int)(mine >> 32), at) << 32) | (unsigned)__shfl((int)mine, at);
    const u64 hit = __ballot(((word >> lane) & 1ull) != 0 && __popcll(word & low_bits(lane)) == k);
    return (c * 64 + at) * WORD + __ffsll((long long)hit) - 1;
}
// All marked pages in front of sequence b's (of the wanted ones).
__device__ __forceinline__ int rank_of(const page_args& a, int b, int lane) {
    int n = 0;
    for (int i = lane; i < b; i += 64) n += (int)a.need[i];
    return __shfl(wave_prefix(n, lane), 63);
}

// The parent whose text sequence b is to take: -1: it stays as it is; -2: it cannot.  A parent stays.
__device__ __forceinline__ int fork_of(const page_args& a, int b) {
    const int p = a.parent[b];
    if (p < 0 || p == b) return -1;
    if (p >= a.batch) return -2;
    const int q = a.parent[p], n = a.seq_len[p];
    if ((q >= 0 && q != p) || n < 1 || (n - 1) / 16 + ((n - 1) % 16 != 0) > a.max_blocks) return -2;
    return p;
}
// The page that it has to have for itself, with the last tokens of the parent's text: -1 if there is none (a full last page, a missing one).
__device__ __forceinline__ int partial_page(const page_args& a, int p) {
    const int cached = a.seq_len[p] - 1;
    if (cached % 16 == 0) return -1;
    const int page = a.table[(size_t)p * a.max_blocks + cached / 16];
    return is_page(a, page) ? page : -1;
}
// The entries of sequence b's row that are to hold pages for positions from from[b] (or the first one that is not cached) to `extra` tokens on.
__device__ __forceinline__ void wanted(const page_args& a, int b, int& lo, int& hi) {
    const int n = a.seq_len[b];
    lo = hi = 0;
    if (n < 1 || a.budget_left[b] <= 0) return;
    const long long end = ((long long)n - 1 + a.extra + 15) / 16;
    lo = (a.from ? max(a.from[b], 0) : n - 1) / 16;
    hi = (int)(end < a.max_blocks ? end : a.max_blocks);
}

enum { INDEX_ONLY, INDEX_FORK, INDEX_RESERVE };
// The index (a workgroup per chunk), and behind it the sequences' needs: a thread (forks) or a wavefront (reserves) per sequence.
template <int MODE>
__global__ __launch_bounds__(256) void pages_index(page_args a) {
    __shared__ int count[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x >= a.chunks) {
        const int at = (int)blockIdx.x - a.chunks;
        if constexpr (MODE == INDEX_FORK) {
            const int b = at * 256 + tid;
            if (b >= a.batch) return;
            const int p = fork_of(a, b);
            if (p == -2) report(a, HS_DEV_PAGE_REFUSED);
            a.need[b] = p >= 0 && partial_page(a, p) >= 0;
        } else if constexpr (MODE == INDEX_RESERVE) {
            const int b = at * 4 + wave;
            if (b >= a.batch) return;
            int lo, hi, n = 0;
            wanted(a, b, lo, hi);
            for (int i = lo + lane; i < hi; i += 64) n += !is_page(a, a.table[(size_t)b * a.max_blocks + i]);
            n = wave_prefix(n, lane);
            if (lane == 63) a.need[b] = (uint32_t)n;
        }
        return;
    }
    const int first = blockIdx.x * CHUNK;
    int ref[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int page = first + (wave * 16 + i) * WORD + lane;
        ref[i] = page < a.n_blocks ? a.refs[page] : 0;
    }
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const u64 held = __ballot(ref[i] != 0);
        const int w = wave * 16 + i;
        if (lane == 0) {
            count[w] = __popcll(held);
            if (blockIdx.x * 64 + w < (unsigned)a.words) a.bits[blockIdx.x * 64 + w] = held;
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int n = count[lane], upto = wave_prefix(n, lane);
        if ((int)blockIdx.x * 64 + lane < a.words) a.before[blockIdx.x * 64 + lane] = (uint32_t)(upto - n);
        if (lane == 63) a.chunk[blockIdx.x] = (uint32_t)upto;
    }
}

// One page less, one more entry on a page.
__device__ __forceinline__ void drop_page(const page_args& a, int page) {
    if (atomicSub(a.refs + page, 1) <= 0) {      // (an entry that nobody counted)
        atomicAdd(a.refs + page, 1);
        report(a, HS_DEV_PAGE_REFUSED);
    }
}

__global__ __launch_bounds__(256) void pages_free(page_args a) {
    const int b = blockIdx.x;
    const int from = a.from[b], to = a.to[b];
    int32_t* row = a.table + (size_t)b * a.max_blocks;
    for (int i = (int)threadIdx.x; i < a.max_blocks; i += 256) {
        if (16ll * i < from || 16ll * i + 16 > to) continue;
        const int page = row[i];
        if (is_page(a, page)) drop_page(a, page);
        if (page != -1) row[i] = -1;
    }
}

// Bytes of a block, by a workgroup of 256: 16 at a time, eight of a thread's on their way.
__device__ __forceinline__ void copy_block(const char* from, char* to, unsigned bytes) {
    const u32x4* src = reinterpret_cast<const u32x4*>(from);
    u32x4* dst = reinterpret_cast<u32x4*>(to);
    const unsigned n = bytes / 16;
    for (unsigned i = threadIdx.x; i < n; i += 256 * 8) {
        u32x4 x[8];
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (i + 256 * u < n) x[u] = __builtin_nontemporal_load(src + i + 256 * u);
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (i + 256 * u < n) __builtin_nontemporal_store(x[u], dst + i + 256 * u);
    }
}
__device__ __forceinline__ void copy_page(const page_args& a, int layer, int from, int to) {
    const size_t at = (size_t)layer * a.n_blocks;
    copy_block(a.k + (at + from) * a.block, a.k + (at + to) * a.block, a.block);
    copy_block(a.v + (at + from) * a.block, a.v + (at + to) * a.block, a.block);
}

// Workgroup b of the first `batch`: sequence b's row of the table, the counts and the rest of its state; behind these one per sequence and
// layer for the copy of the partial page.  (A child's copy needs nothing of its row, and its parent's row stays.)
__global__ __launch_bounds__(256) void pages_fork(page_args a) {
    __shared__ int s_page;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool copies = (int)blockIdx.x >= a.batch;
    const int b = copies ? ((int)blockIdx.x - a.batch) / a.layers : (int)blockIdx.x;
    const int p = fork_of(a, b);
    if (p < 0) return;
    const int src = partial_page(a, p);
    if (copies && src < 0) return;
    if (wave == 0 && src >= 0) {
        const int page = select_page<true>(a, rank_of(a, b, lane), lane);
        if (lane == 0) s_page = page;
    }
    __syncthreads();
    const int own = src >= 0 ? s_page : -1;
    if (src >= 0 && own < 0) {      // no page is left: the sequence stays as it is
        if (!copies && tid == 0) report(a, HS_DEV_PAGES_EXHAUSTED);
        return;
    }
    if (copies) {
        copy_page(a, ((int)blockIdx.x - a.batch) % a.layers, src, own);
        return;
    }
    const int n = a.seq_len[p], full = (n - 1) / 16;
    int32_t* row = a.table + (size_t)b * a.max_blocks;
    const int32_t* of = a.table + (size_t)p * a.max_blocks;
    for (int i = tid; i < a.max_blocks; i += 256) {
        const int old = row[i], page = i < full ? of[i] : i == full ? own : -1, now = is_page(a, page) ? page : -1;
        if (now == old) continue;
        if (now >= 0) atomicAdd(a.refs + now, 1);
        if (is_page(a, old)) drop_page(a, old);
        row[i] = now;
    }
    for (int i = tid; i < a.w_max; i += 256) a.tail[(size_t)b * a.w_max + i] = a.tail[(size_t)p * a.w_max + i];
    if (a.tokens)
        for (int i = tid; i < min(n, a.tokens_stride); i += 256)
            a.tokens[(size_t)b * a.tokens_stride + i] = a.tokens[(size_t)p * a.tokens_stride + i];
    if (tid == 0) {
        a.seq_len[b] = n;
        a.tail_len[b] = a.tail_len[p];
        a.k_state[b] = a.k_state[p];
        a.budget_left[b] = a.budget_left[p];
    }
}

// A wavefront per sequence takes the free pages from its rank on: a chunk's words at a time, a word's bits by the lanes.
__global__ __launch_bounds__(64) void pages_reserve(page_args a) {
    __shared__ int list[2 * WORD];      // pages at hand; a word adds up to 64 to fewer than 64
    const int b = blockIdx.x, lane = threadIdx.x;
    if (a.need[b] == 0) return;
    int lo, hi;
    wanted(a, b, lo, hi);
    int32_t* row = a.table + (size_t)b * a.max_blocks;
    int r = rank_of(a, b, lane), have = 0;
    int c = find_chunk<true>(a, r, lane);
    u64 mine = 0;
    auto load_chunk = [&]() { mine = c < a.chunks && c * 64 + lane < a.words ? marked<true>(a, c * 64 + lane) : 0ull; };
    if (c >= 0) {
        load_chunk();
        // those of other sequences: r pages of the chunk
        const int n = __popcll(mine), skip = r - (wave_prefix(n, lane) - n);
        if (skip >= n) mine = 0;
        else
            for (int i = 0; i < skip; i++) mine &= mine - 1;
    }
    for (int i0 = lo; i0 < hi; i0 += 64) {
        const int i = i0 + lane;
        const bool missing = i < hi && !is_page(a, row[i]);
        const u64 all = __ballot(missing);
        const int want = __popcll(all), at = __popcll(all & low_bits(lane));
        while (have < want && c >= 0 && c < a.chunks) {
            const u64 some = __ballot(mine != 0);
            if (!some) {
                c++;
                load_chunk();
                continue;
            }
            const int w = __ffsll((long long)some) - 1;
            const u64 word = ((u64)(unsigned)__shfl((int)(mine >> 32), w) << 32) | (unsigned)__shfl((int)mine, w);
            if ((word >> lane) & 1ull) list[have + __popcll(word & low_bits(lane))] = (c * 64 + w) * WORD + lane;
            if (lane == w) mine = 0;
            have += __popcll(word);
        }
        __syncthreads();
        if (missing) {
            if (at < have) {
                row[i] = list[at];
                a.refs[list[at]] = 1;
            } else {
                row[i] = -1;
                report(a, HS_DEV_PAGES_EXHAUSTED);
            }
        }
        const int left = max(0, have - want), keep = lane < left ? list[want + lane] : 0;
        __syncthreads();
        if (lane < left) list[lane] = keep;
        have = left;
        __syncthreads();
    }
}

// Held pages in front of page e (e <= n_blocks), and the r-th free page: by one thread.  chunk[] as prefix sums in `upto` (LDS, or memory).
__device__ __forceinline__ int held_before(const page_args& a, const int* sums, int e) {
    const int w = e / WORD;
    if (w >= a.words) return sums[a.chunks];
    return sums[w / 64] + (int)a.before[w] + __popcll(a.bits[w] & low_bits(e % WORD));
}
__device__ __forceinline__ int free_page(const page_args& a, const int* sums, int r) {
    int lo = 0, hi = a.chunks - 1;      // the last chunk with at most r free pages in front of it
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (mid * CHUNK - sums[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    r -= lo * CHUNK - sums[lo];
    int w = lo * 64, last = min(w + 63, a.words - 1);
    while (w < last) {
        const int mid = (w + last + 1) / 2;
        if (marked_before<true>(a, mid) <= r) w = mid;
        else last = mid - 1;
    }
    r -= marked_before<true>(a, w);
    const u64 word = marked<true>(a, w);
    int bit = 0;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1)
        if (__popcll(word & low_bits(bit + s)) <= r) bit += s;
    return w * WORD + bit;
}

// Small pools: one workgroup has the index in LDS and needs no launch for it.  (16384 pages: 16 of a thread's counts are on their way at once.)
constexpr int SMALL_PAGES = 16384, SMALL_WORDS = SMALL_PAGES / WORD, SMALL_CHUNKS = SMALL_PAGES / CHUNK;
struct small_index {
    u64 bits[SMALL_WORDS];
    uint32_t before[SMALL_WORDS], chunk[SMALL_CHUNKS];
    int sums[SMALL_CHUNKS + 1];
};
// By 1024 threads; a's index is this one then.  between(): what is done while the counts are on their way.
template <typename Between>
__device__ __forceinline__ void build_small(page_args& a, small_index& x, Between between) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int ref[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int page = (wave * 16 + i) * WORD + lane;
        ref[i] = page < a.n_blocks ? a.refs[page] : 0;
    }
    hs_loads_issued();
    between();
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const u64 held = __ballot(ref[i] != 0);
        if (lane == 0) {
            x.bits[wave * 16 + i] = held;
            x.before[wave * 16 + i] = (uint32_t)__popcll(held);
        }
    }
    __syncthreads();
    if (wave < SMALL_CHUNKS) {
        const int n = (int)x.before[wave * 64 + lane], upto = wave_prefix(n, lane);
        x.before[wave * 64 + lane] = (uint32_t)(upto - n);
        if (lane == 63) x.chunk[wave] = (uint32_t)upto;
    }
    __syncthreads();
    if (tid <= SMALL_CHUNKS) {
        int sum = 0;
        for (int c = 0; c < tid; c++) sum += (int)x.chunk[c];
        x.sums[tid] = sum;
    }
    __syncthreads();
    a.bits = x.bits;
    a.before = x.before;
    a.chunk = x.chunk;
}

// A few pages per sequence: a thread per sequence counts what it lacks, and takes what is free from its place on.  (Turnovers of 117 sequences and 2343
// pages with a launch for the index and one of a wavefront per sequence: 64 us, with this one 61; of 4 sequences 18 and 15.)
constexpr int SMALL_BATCH = 1024, SMALL_EXTRA = 48, SMALL_ENTRIES = (15 + SMALL_EXTRA + 15) / 16;
__global__ __launch_bounds__(1024) void pages_reserve_small(page_args a) {
    __shared__ small_index x;
    __shared__ int waves[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int lo = 0, hi = 0, n = 0, r = 0;
    bool missing[SMALL_ENTRIES] = {};
    int32_t* row = a.table + (size_t)min(tid, a.batch - 1) * a.max_blocks;
    build_small(a, x, [&] {
        if (tid < a.batch) {
            wanted(a, tid, lo, hi);
            int page[SMALL_ENTRIES];
#pragma unroll
            for (int i = 0; i < SMALL_ENTRIES; i++) page[i] = lo + i < hi ? row[lo + i] : 0;
#pragma unroll
            for (int i = 0; i < SMALL_ENTRIES; i++) {
                missing[i] = lo + i < hi && !is_page(a, page[i]);
                n += missing[i];
            }
        }
        r = wave_prefix(n, lane);
        if (lane == 63) waves[wave] = r;
        r -= n;
    });
    for (int w = 0; w < wave; w++) r += waves[w];
    const int free = a.n_blocks - x.sums[a.chunks];
#pragma unroll
    for (int i = 0; i < SMALL_ENTRIES; i++) {
        if (!missing[i]) continue;
        const int page = r < free ? free_page(a, x.sums, r) : -1;
        r++;
        row[lo + i] = page;
        if (page >= 0) a.refs[page] = 1;
        else report(a, HS_DEV_PAGES_EXHAUSTED);
    }
}

// Every page's number after the move: the k-th free page below n_live is taken by the k-th held one from n_live on.
__device__ __forceinline__ void map_page(const page_args& a, const int* sums, int page) {
    const int live = sums[a.chunks], low = held_before(a, sums, live);
    if (page == 0) {
        *a.n_moves = live - low;
        if (a.n_live) *a.n_live = live;
    }
    int to = -1;
    if ((a.bits[page / WORD] >> (page % WORD)) & 1ull) {
        to = page;
        if (page >= live) {
            const int k = held_before(a, sums, page) - low;
            to = free_page(a, sums, k);
            a.pairs[2 * k] = page;
            a.pairs[2 * k + 1] = to;
            a.refs[to] = a.refs[page];
            a.refs[page] = 0;
        }
    }
    a.moved[page] = to;
}
__global__ __launch_bounds__(1024) void pages_map_small(page_args a) {
    __shared__ small_index x;
    build_small(a, x, [] {});
    for (int page = threadIdx.x; page < a.n_blocks; page += 1024) map_page(a, x.sums, page);
}
constexpr int CHUNKS_MAX = HS_PAGES_MAX / CHUNK;
__global__ __launch_bounds__(256) void pages_map(page_args a) {
    __shared__ int sums[CHUNKS_MAX + 1];
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) {
        int carry = 0;
        for (int c0 = 0; c0 < a.chunks; c0 += 64) {
            const int n = marked_in_chunk<false>(a, c0 + lane), upto = carry + wave_prefix(n, lane);
            if (c0 + lane < a.chunks) sums[c0 + lane] = upto - n;
            carry = __shfl(upto, 63);
        }
        if (lane == 0) sums[a.chunks] = carry;
    }
    __syncthreads();
    const int page = blockIdx.x * 256 + tid;
    if (page < a.n_blocks) map_page(a, sums, page);
}
// The tables' entries (the first max_batch workgroups) and the pages themselves, a run of (page, layer) each.
__global__ __launch_bounds__(256) void pages_move(page_args a) {
    const int rows = a.max_rows;
    if ((int)blockIdx.x < rows) {
        int32_t* row = a.table + (size_t)blockIdx.x * a.max_blocks;
        for (int i = (int)threadIdx.x; i < a.max_blocks; i += 256) {
            const int page = row[i];
            if (!is_page(a, page)) continue;
            const int to = a.moved[page];
            if (to >= 0 && to != page) row[i] = to;
        }
        return;
    }
    const long long items = (long long)*a.n_moves * a.layers;
    const int at = (int)blockIdx.x - rows, of = (int)gridDim.x - rows;
    for (long long i = items * at / of; i < items * (at + 1) / of; i++) {
        const int k = (int)(i / a.layers);
        copy_page(a, (int)(i % a.layers), a.pairs[2 * k], a.pairs[2 * k + 1]);
    }
}

page_args make_args(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_page_pool* pool) {
    page_args a = {};
    a.refs = pool->refs;
    a.table = pool->table;
    a.n_blocks = cache->n_blocks;
    a.max_blocks = ctx->lim.max_blocks_per_seq;
    a.words = (cache->n_blocks + WORD - 1) / WORD;
    a.chunks = (a.words + 63) / 64;
    a.max_rows = ctx->lim.max_batch;
    char* at = (char*)pool->scratch;
    auto take = [&](size_t bytes) { char* p = at; at += (bytes + 15) / 16 * 16; return p; };
    a.bits = (u64*)take((size_t)a.words * 8);
    a.before = (uint32_t*)take((size_t)a.words * 4);
    a.chunk = (uint32_t*)take((size_t)a.chunks * 4);
    a.need = (uint32_t*)take((size_t)ctx->lim.max_batch * 4);
    a.pairs = (int32_t*)take((size_t)cache->n_blocks * 4 + 8);      // (at most n_blocks / 2 pages move)
    a.moved = (int32_t*)take((size_t)cache->n_blocks * 4);
    a.n_moves = (int32_t*)take(16);
    a.w_max = ctx->lim.w_max;
    a.k = (char*)cache->k;
    a.v = (char*)cache->v;
    a.block = (unsigned)ctx->desc.n_kv_heads * 16 * ctx->desc.head_dim * (hs_fp32_activations(ctx) ? 4 : 2);
    a.layers = ctx->desc.n_layers;
    a.err = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.err);
    if (seq) {
        a.batch = seq->batch;
        a.seq_len = seq->seq_len;
        a.tail = seq->tail;
        a.tail_len = seq->tail_len;
        a.k_state = seq->k_state;
        a.budget_left = seq->budget_left;
        a.tokens = seq->tokens;
        a.tokens_stride = seq->tokens_stride;
    }
    return a;
}

}  // namespace

size_t hs_pages_scratch(const hs_ctx* ctx, int n_blocks) {
    auto up = [](size_t n) { return (n + 15) / 16 * 16; };
    const size_t words = ((size_t)n_blocks + WORD - 1) / WORD, chunks = (words + 63) / 64;
    return up(words * 8) + up(words * 4) + up(chunks * 4) + up((size_t)ctx->lim.max_batch * 4) + up((size_t)n_blocks * 4 + 8) + up((size_t)n_blocks * 4) + 16;
}

void hs_launch_pages_free(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_page_pool* pool, const int32_t* from,
                          const int32_t* to, hipStream_t st) {
    page_args a = make_args(ctx, cache, seq, pool);
    a.from = from;
    a.to = to;
    hipLaunchKernelGGL(pages_free, dim3(a.batch), dim3(256), 0, st, a);
}

void hs_launch_pages_fork(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_page_pool* pool, const int32_t* parent,
                          hipStream_t st) {
    page_args a = make_args(ctx, cache, seq, pool);
    a.parent = parent;
    hipLaunchKernelGGL((pages_index<INDEX_FORK>), dim3(a.chunks + (a.batch + 255) / 256), dim3(256), 0, st, a);
    hipLaunchKernelGGL(pages_fork, dim3(a.batch * (1 + a.layers)), dim3(256), 0, st, a);
}

void hs_launch_pages_reserve(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_page_pool* pool, const int32_t* from, int extra,
                             hipStream_t st) {
    page_args a = make_args(ctx, cache, seq, pool);
    a.from = from;
    a.extra = extra;
    if (!from && extra <= SMALL_EXTRA && a.batch <= SMALL_BATCH && a.n_blocks <= SMALL_PAGES) {
        hipLaunchKernelGGL(pages_reserve_small, dim3(1), dim3(1024), 0, st, a);
        return;
    }
    hipLaunchKernelGGL((pages_index<INDEX_RESERVE>), dim3(a.chunks + (a.batch + 3) / 4), dim3(256), 0, st, a);
    hipLaunchKernelGGL(pages_reserve, dim3(a.batch), dim3(64), 0, st, a);
}

void hs_launch_pages_compact(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_page_pool* pool, int32_t* n_live, int32_t* moved, hipStream_t st) {
    page_args a = make_args(ctx, cache, nullptr, pool);
    a.n_live = n_live;
    if (moved) a.moved = moved;
    if (a.n_blocks <= SMALL_PAGES) {
        hipLaunchKernelGGL(pages_map_small, dim3(1), dim3(1024), 0, st, a);
    } else {
        hipLaunchKernelGGL((pages_index<INDEX_ONLY>), dim3(a.chunks), dim3(256), 0, st, a);
        hipLaunchKernelGGL(pages_map, dim3((a.n_blocks + 255) / 256), dim3(256), 0, st, a);
    }
    const long long most = (long long)a.n_blocks / 2 * a.layers, wide = 8ll * ctx->n_cu;
    hipLaunchKernelGGL(pages_move, dim3((unsigned)(a.max_rows + std::max(1ll, std::min(most, wide)))), dim3(256), 0, st, a);
}
