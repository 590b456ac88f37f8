// Paged attention with a sliding window and sinks: a query row at position p sees, of the keys that it would see without
// a window (the cached ones and its ancestors among the draft's nodes, or the tokens of its chunk up to itself), those at
// positions t > p - window and those at t < sinks.
//
//   out[row, h] = sum_t softmax_t(q[row, h] . k[t, h / G] / sqrt(head_dim)) v[t, h / G]  over the visible t; 0 if there is none
//
// A sequence of L cached tokens and nn rows needs the keys [0, sinks) and [L + 1 - window, L + nn), whatever its length: only
// their pages are looked up and read.  (Of a sequence that has outgrown its block table, what of these lies in the table.)
//
// Scores are computed transposed, S^T = K . Q^T (v_mfma_f32_32x32x16_bf16), for 32 query rows (rows of one token's G query heads, which share a
// KV head, are neighbours) and 32 keys at a time, so that a lane has the scores of one query row and the softmax statistics are its own scalars.
// The second product O^T = V^T . P^T takes 16 tokens of V^T, which the cache holds token index fastest: a lane's operand is 16 contiguous bytes,
// tokens 8 half .. 8 half + 7 of a page.  The rows of the first product's operand are therefore the page's keys in the order of page_order, which
// leaves a lane exactly the probabilities of those tokens.
//
// A draft's rows are few and its keys many, and memory bounds it.  Four row tiles share a stream of key tiles through LDS; a workgroup walks all
// keys of a (sequence, KV head), or a run of partitions, whose results a launch of its own joins (see plan_rows).  128 single tokens, 28 heads,
// 1024 keys: 51 us, 5.3 TB/s (a copy reaches 4.9); 256 drafts, 4096 keys: 362 us, 5.2 TB/s; 64 trees of 17 nodes, 40 heads, 2048 keys: 97 us, 5.8
// TB/s; the stream alone, without products, 319 and 95 us when these took 412 and 131.  A chunk's rows are many: a workgroup takes 128 of them
// through all their keys (512 tokens each of 7 sequences and 257 of an eighth, 28 heads, 1024 keys: 89 us, 637 TFLOP/s of the 1215 that a large product
// of matrices reaches; matrix unit, vector unit and LDS are each busy for two fifths of the time, with two wavefronts per SIMD to overlap them).
//
// Every sum has an order that depends on absolute key positions only (32-key tiles, partitions of part_keys, if any, merged in index order;
// keys that a row does not see contribute exact zeros): a row's result does not depend on what other rows are computed with it.
#include <algorithm>

#include "hs_attention_ring.h"
#include "hs_internal.h"

using namespace hs_ring;

namespace {

struct win_args {
    const bf16_t *q, *kc, *vc;          // kc, vc: at the layer
    const int32_t *seq_len, *block_table, *row_off, *row2seq, *pos;
    const uint64_t* anc_mask;
    bf16_t* out;
    _Float16* part_o;
    float* part_ml;
    int batch, max_blocks, n_blocks, hq, hkv, window, sinks, part_keys, max_parts, groups, kind;
    size_t part_rows;                   // rows of partial results of a partition: those of the limits' rows and all heads
    float scale_log2, lag;
};

// The keys that a sequence's rows need: [0, sink_end) and [first, total), and the partitions of the key axis that hold them: n_sink
// from the axis's start, then those from p_first on.  (Keys beyond the block table do not exist.)
struct win_span {
    int L, total, first, sink_end, n_sink, p_first, n_parts;
    __device__ __forceinline__ int partition(int c) const { return c < n_sink ? c : p_first + (c - n_sink); }
    // where a walk that has come to kb goes on
    __device__ __forceinline__ int skip(int kb) const { return kb >= sink_end && kb + 32 <= first ? first & ~31 : kb; }
};
__device__ __forceinline__ win_span make_span(int seq_len, int nn, const win_args& a) {
    const int cap = a.max_blocks * 16;
    win_span s;
    // (A sequence may have outgrown its table: its windows lie where its positions are, and only the walk ends with the table.  The bound keeps
    // sums with L in 32 bits: hs_create takes no more rows than 2^25.)
    s.L = min(seq_len - 1, INT32_MAX - (1 << 25));
    s.total = min(s.L + nn, cap);
    s.first = max(0, s.L + 1 - a.window);
    s.sink_end = min(min(a.sinks, s.first), s.total);
    s.n_sink = (s.sink_end + a.part_keys - 1) / a.part_keys;
    s.p_first = max(s.first / a.part_keys, s.n_sink);
    // Each of them has a key, so that a walk over all keys comes through all of them.  (A sequence that has outgrown its table may have no
    // key in its window.  No more than there is room for: a draft of more nodes than the limits allow is not laid out by anybody.)
    const int n_window = s.first < s.total ? max(0, (s.total + a.part_keys - 1) / a.part_keys - s.p_first) : 0;
    s.n_parts = s.L < 0 || nn <= 0 ? 0 : min(a.max_parts, s.n_sink + n_window);
    return s;
}


// Walks keys k0, ... (32 at a time, k_end excluded) with one row tile.  all_lo, all_hi: every row sees the keys in [all_lo, all_hi) and
// in [0, min(sinks, all_hi)).
template <int HD>
__device__ __forceinline__ bool walk_keys(const win_args& a, const win_span& s, const int32_t* __restrict__ bt, int j, int k0, int k_end,
                                          int all_lo, int all_hi, row_tile<HD>& t, int lane) {
    constexpr int NKS = HD / 16, NDT = HD / 32;
    const int half = lane >> 5, l32 = lane & 31;
    const size_t page_elems = (size_t)a.hkv * 16 * HD;
    const bf16_t* kp = a.kc + (size_t)j * 16 * HD + page_order(l32 & 15) * HD + half * 8;
    const bf16_t* vp = a.vc + (size_t)j * 16 * HD + l32 * 16 + half * 8;

    // lane i holds the page of keys 1024 n + 16 i .. + 15: -1 where no row sees any of them, or the table has none
    int held = -1, my_page = -1;
    auto hold = [&](int kb) {
        if ((kb >> 10) == held) return;
        held = kb >> 10;
        const int at = held * 64 + lane, p0 = at * 16;
        my_page = -1;
        if (at < a.max_blocks && p0 < k_end && (p0 < s.sink_end || p0 + 16 > s.first)) my_page = bt[at];
        if (my_page >= a.n_blocks) my_page = -1;
    };
    auto find = [&](int kb) -> places {
        hold(kb);
        return {__builtin_amdgcn_readlane(my_page, (kb >> 4) & 63), __builtin_amdgcn_readlane(my_page, ((kb >> 4) & 63) + 1)};
    };
    auto load_k = [&](const places& p, key_tile<HD>& k) {
        // (a page that does not exist: some other, of which nothing is used)
        const bf16_t* src = kp + (size_t)max(l32 < 16 ? p.p0 : p.p1, 0) * page_elems;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) k.k[ks] = *reinterpret_cast<const bf16x8*>(src + ks * 16);
    };
    auto load_v = [&](const places& p, value_tile<HD>& v) {
#pragma unroll
        for (int pp = 0; pp < 2; pp++) {
            const bf16_t* src = vp + (size_t)max(pp ? p.p1 : p.p0, 0) * page_elems;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)      // (non-temporal: a line of V is one load's, a line of K several loads')
                v.v[pp][dt] = __builtin_bit_cast(bf16x8, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + dt * 32 * 16)));
        }
    };

    bool odd = false;
    if (k0 >= k_end) return odd;
    key_tile<HD> k;
    value_tile<HD> v;
    places cur = find(k0);
    load_k(cur, k);
    load_v(cur, v);
    for (int kb = k0;;) {
        const int next = s.skip(kb + 32);
        const bool more = next < k_end;
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; e++) sc[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.k[ks], t.qf[ks], sc, 0, 0, 0);
        const places here = cur;
        if (more) {
            cur = find(next);
            load_k(cur, k);
        }
        bf16x8 pb[2];
        const bool masked = tile_masked(a, here, kb, all_lo, all_hi);
        const float alpha = take_scores<HD>(a, s, t, sc, here, masked, kb, half);
        take_probabilities<HD>(a, t, sc, alpha, pb);
        if (masked) odd |= mask_values<HD>(v);
        take_values<HD>(t, v, pb);
        if (!more) return __any(odd);
        load_v(cur, v);
        kb = next;
    }
}

// Queries and visible keys of a draft's row tile.
template <int HD>
__device__ __forceinline__ void load_rows(const win_args& a, const win_span& s, int r0, int nn, int rt, int j, int all_lo, row_tile<HD>& t,
                                          int lane) {
    const int half = lane >> 5, l32 = lane & 31, G = a.hq / a.hkv, R = nn * G, rho = rt * 32 + l32;
    load_query_tile<HD>(a.q, a.anc_mask, r0, rt, R, G, a.hq, j, half, l32, t.qf, t.anc);
    const int pos = rho < R ? max(a.pos[r0 + rho / G], 0) : s.L;
    t.lo = min(max(pos + 1 - a.window, s.first), all_lo);
    t.hi = s.L;
    if (a.window < HS_MAX_NODES) {
        // ancestors that lie behind the window
        uint64_t left = t.anc;
        for (uint64_t todo = t.anc; todo; todo &= todo - 1) {
            const int i = __ffsll((unsigned long long)todo) - 1;
            const int at = i < nn ? a.pos[r0 + i] : -1;
            if (i >= nn || !(at > pos - a.window || at < a.sinks)) left &= ~(1ull << i);
        }
        t.anc = left;
    }
}

// Partitions c, c + step, ... of a (sequence, KV head) by one wavefront.
template <int HD>
__device__ __forceinline__ void walk_partitions(const win_args& a, const win_span& s, const int32_t* __restrict__ bt, int j, int r0, int nn,
                                                int c, int step, int lane) {
    const int G = a.hq / a.hkv, R = nn * G;
    // its depth is below nn, so that from all_lo on every row sees every cached key
    const int all_lo = max(0, s.L + nn - a.window);
    // (of a draft with more nodes than the limits allow there are more tiles, and more partitions)
    for (; c < s.n_parts; c += step)
        for (int rt = 0; rt * 32 < R; rt++) {
            row_tile<HD> t;
            load_rows<HD>(a, s, r0, nn, rt, j, all_lo, t, lane);
            begin_tile<HD>(t);
            const int p = s.partition(c);
            const int k0 = s.skip(p * a.part_keys), k_end = min(s.total, (p + 1) * a.part_keys);
            if (walk_keys<HD>(a, s, bt, j, k0, k_end, all_lo, s.L, t, lane)) add_odd<HD>(a, s, bt, j, k0, k_end, all_lo, s.L, t, lane);
            put_partial<HD>(a, t, r0, rt, R, G, j, c, lane);
        }
}

// Small calls of at most 32 query rows per KV head (plain decoding): a wavefront per partition.
template <int HD>
__global__ __launch_bounds__(256, 2) void window_rows(win_args a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x % a.groups, pair = blockIdx.x / a.groups;
    const int j = pair % a.hkv, b = pair / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0;
    const win_span s = make_span(a.seq_len[b], nn, a);
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    walk_partitions<HD>(a, s, bt, j, r0, nn, 4 * g + wave, 4 * a.groups, lane);
}


// Drafts of any size.  A workgroup takes all keys (WHOLE) or a run of partitions of a (sequence, KV head) with four row tiles.  (A sequence with
// one row tile keeps one wavefront busy with products: two workgroups per compute unit are enough for the memory's pace.)
// There are one or two groups of four tiles (at most 256 query rows per KV head); the workgroups of the second, most of which have nothing to do,
// come last.  (In turn with the others, live and idle workgroups alternated on the way to the shader engines, and of two places on a compute unit
// one stayed empty: 256 sequences with a long tail of lengths, 4096 keys, 28 heads, 600 us instead of 435.)
constexpr int WIN_START = 3;
template <int HD, bool WHOLE>
__global__ __launch_bounds__(256, 2) void window_rows_ring(win_args a, int tile_groups) {
    __shared__ __attribute__((aligned(1024))) win_lds<HD> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = a.groups * a.hkv * a.batch, unit = blockIdx.x % units, group = blockIdx.x / units;
    const int g = unit % a.groups, pair = unit / a.groups;
    const int j = pair % a.hkv, b = pair / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0;
    const int G = a.hq / a.hkv, R = nn * G, nrt = (R + 31) >> 5;
    const win_span s = make_span(a.seq_len[b], nn, a);
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    const int all_lo = max(0, s.L + nn - a.window);      // (see walk_partitions)
    const int c_begin = (int)((long long)s.n_parts * g / a.groups), c_end = (int)((long long)s.n_parts * (g + 1) / a.groups);
    if (4 * group >= nrt || (!WHOLE && c_begin >= c_end)) return;
    const int k0 = s.skip(WHOLE ? 0 : s.partition(c_begin) * a.part_keys);
    const int k_end = !WHOLE ? min(s.total, (s.partition(c_end - 1) + 1) * a.part_keys)
                             : s.n_parts > 0 ? min(s.total, s.L + HS_MAX_NODES) : 0;      // (no row sees a slot beyond those of 64 nodes)
    // (one turn, but for a draft of more nodes than the launch provides for)
    for (int tg = 4 * group; tg < nrt; tg += 4 * tile_groups) {
        const int rt = tg + ((wave - g - j - b) & 3);      // (two of four wavefronts with rows are not the same two everywhere)
        int c = c_begin;
        row_tile<HD> t;
        load_rows<HD>(a, s, r0, nn, rt, j, all_lo, t, lane);
        begin_tile<HD>(t);
        if constexpr (WHOLE) {
            ring_keys<HD, false>(a, s, bt, j, k0, k_end, INT32_MAX / 2, all_lo, s.L, t, rt >= nrt, lds, [&]() __attribute__((always_inline)) {});
            put_result<HD>(a, t, r0, rt, R, G, j, lane);
        } else {
            ring_keys<HD, false>(a, s, bt, j, k0, k_end, a.part_keys, all_lo, s.L, t, rt >= nrt, lds, [&]() __attribute__((always_inline)) {
                put_partial<HD>(a, t, r0, rt, R, G, j, c, lane);
                begin_tile<HD>(t);
                c++;
            });
        }
    }
}

// Joins the partitions of a row's query heads in their order: a wavefront takes 512 / HD heads of a row, a lane eight elements of one.  Eight
// partitions at a time, all of which are asked for before the first is used; more than eight (in steps of eight) move the maximum as a
// softmax over the keys does.  EARLY: with few rows the first eight are asked for before it is known how many there are, and whether there is
// the row: what a launch of a few rows takes is its chain of round trips to memory (count, row's sequence, its length, partial results).
template <int HD, bool EARLY>
__global__ __launch_bounds__(256) void window_merge(win_args a) {
    constexpr int LANES = HD / 8, HEADS = 64 / LANES, AHEAD = 8;
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63, head = (blockIdx.y * 4 + (threadIdx.x >> 6)) * HEADS + lane / LANES;
    if ((blockIdx.y * 4 + (threadIdx.x >> 6)) * HEADS >= a.hq) return;
    for (int row = blockIdx.x; (size_t)row * a.hq < a.part_rows; row += gridDim.x) {
        const size_t prow = (size_t)row * a.hq + min(head, a.hq - 1);
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + prow;
        const _Float16* po = a.part_o + prow * HD + 8 * (lane % LANES);
        float2 x0[AHEAD];
        f16x8 v0[AHEAD];
        if constexpr (EARLY) {
            // (in bounds whether the row and its partitions exist or not: the loop goes no further than the workspace's rows)
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                x0[p] = ml[min(p, a.max_parts - 1) * a.part_rows];
                v0[p] = *reinterpret_cast<const f16x8*>(po + min(p, a.max_parts - 1) * a.part_rows * HD);
            }
            hs_loads_issued();
        }
        if (row >= a.row_off[a.batch]) return;
        const int b = a.row2seq[row];
        const int n = make_span(a.seq_len[b], a.row_off[b + 1] - a.row_off[b], a).n_parts;
        float top = -INFINITY, den = 0.f, acc[8];
#pragma unroll
        for (int i = 0; i < 8; i++) acc[i] = 0.f;
        for (int p0 = 0; p0 < n; p0 += AHEAD) {
            float2 x[AHEAD];
            f16x8 v[AHEAD];
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                const int at = min(p0 + p, n - 1);
                if (EARLY && p0 == 0) {
                    x[p] = p < n ? x0[p] : make_float2(-INFINITY, 0.f);
                    v[p] = v0[p];
                } else {
                    x[p] = ml[at * a.part_rows];
                    v[p] = *reinterpret_cast<const f16x8*>(po + at * a.part_rows * HD);
                }
            }
            float m = top;
#pragma unroll
            for (int p = 0; p < AHEAD; p++) m = fmaxf(m, x[p].x);
            const float safe = m == -INFINITY ? 0.f : m;
            if (p0 > 0) {
                const float alpha = fast_exp2(top - safe);
                den *= alpha;
#pragma unroll
                for (int i = 0; i < 8; i++) acc[i] *= alpha;
            }
            top = m;
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                if (p0 + p >= n) break;
                // the partition's weight in the whole; its output is stored normalised
                const float w = fast_exp2(x[p].x - safe) * x[p].y;
                den += w;
#pragma unroll
                for (int i = 0; i < 8; i++) acc[i] += w * (float)v[p][i];
            }
        }
        if (head < a.hq) {
            const float inv = den == 0.f ? 0.f : 1.f / den;
            u32x4 y;
#pragma unroll
            for (int i = 0; i < 4; i++) y[i] = (uint32_t)to_bf16(acc[2 * i] * inv) | ((uint32_t)to_bf16(acc[2 * i + 1] * inv) << 16);
            *reinterpret_cast<u32x4*>(a.out + ((size_t)row * a.hq + head) * HD + 8 * (lane % LANES)) = y;
        }
    }
}

// The rows of a chunk: consecutive tokens, row i of a sequence at position L + i.  A workgroup takes 128 query rows of one (sequence, KV
// head), a wavefront 32 of them, through all their keys: with hundreds of rows per sequence there is enough to do without cutting the key axis.
// (Every wavefront with the keys of its own 32 rows, from the caches into registers: 165 us for 8 x 512 tokens, 28 heads, 1024 keys.)
template <int HD>
__global__ __launch_bounds__(256, 2) void window_chunk(win_args a, int nx) {
    __shared__ __attribute__((aligned(1024))) win_lds<HD> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    // Ids are dealt round-robin to the eight XCDs: with a multiple of eight pairs, all blocks of a pair go to one XCD and find its K and V in
    // that L2.
    const int pairs = a.hkv * a.batch;
    int pair = blockIdx.x / nx, bx = blockIdx.x % nx;
    if ((pairs & 7) == 0) {
        const int local = blockIdx.x >> 3;
        pair = (local / nx) * 8 + (blockIdx.x & 7);
        bx = local % nx;
    }
    const int j = pair % a.hkv, b = pair / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0;
    win_span s = make_span(a.seq_len[b], nn, a);
    if (nn <= 0) return;
    const int G = a.hq / a.hkv, R = nn * G;
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    for (; bx * 128 < R; bx += nx) {
        // the keys of the block's rows
        s.first = max(0, s.L + bx * 128 / G + 1 - a.window);
        s.sink_end = min(min(a.sinks, s.first), s.total);
        const int k_end = min(s.total, s.L + min(nn - 1, (bx * 128 + 127) / G) + 1);
        const int rt = bx * 4 + wave, rho = rt * 32 + l32;
        const int node0 = rt * 32 / G, node1 = min(nn - 1, (rt * 32 + 31) / G), node = min(rho / G, nn - 1);
        row_tile<HD> t;
        load_query_tile<HD>(a.q, nullptr, r0, rt, R, G, a.hq, j, half, l32, t.qf, t.anc);
        t.lo = max(0, s.L + node + 1 - a.window);
        t.hi = s.L + node + 1;
        begin_tile<HD>(t);
        ring_keys<HD, true>(a, s, bt, j, s.skip(0), k_end, INT32_MAX / 2, max(0, s.L + node1 + 1 - a.window), s.L + node0 + 1, t, rt * 32 >= R, lds,
                      [&]() __attribute__((always_inline)) {});
        put_result<HD>(a, t, r0, rt, R, G, j, lane);
    }
}

// The most query rows per KV head that a draft can have.
int rows_of(const hs_ctx* ctx) { return ctx->desc.n_q_heads / ctx->desc.n_kv_heads * (1 + ctx->lim.c_max * ctx->lim.k_max); }

// How a draft's keys are taken.  A function of the context's limits, the window and the sinks, so that the order of a row's sums is the same in
// every step.
//
// WIN_WHOLE: a workgroup per (sequence, KV head), which writes the result itself.  Where there are as many of these as compute units: partial
// results in the middle of the key stream and the launch that joins them cost 256 drafts of 28 heads over 4096 keys 408 instead of 365 us, 64
// trees of 40 heads over 2048 keys 130 instead of 101, 64 single tokens of 28 heads over 1024 keys 51 instead of 38, 64 drafts of 28 heads over
// 4096 keys 119 instead of 117.  The limits do not say how many sequences there are now: 8 drafts within limits for 256 take 108 us instead of
// 60.  Only up to 16000 keys, since a workgroup walks all that a sequence has (and its pages' numbers lie in LDS): texts of 2048 to 16384 tokens, 128
// drafts of 28 heads over 8000 keys 317 us instead of 398, 15000 keys 494 and 589; 64 drafts behind up to 20000 tokens 197 and 225, 354 and 334.
// With fewer sequences, too, where the walk is shorter than a second launch takes (8 single tokens over 68 keys 13.1 us instead of 14.7, 128 keys
// 14.4 and 15.1, 256 keys 17.4 and 15.4; 8 drafts 13.2 and 15.4, 14.3 and 16.2, 17.4 and 17.2).
//
// WIN_FEW: a wavefront per partition, of limits with at most 32 query rows per KV head and two tiles of 32 keys for every SIMD: all of them are
// on their way at once (8 single tokens of 28 heads over 1024 keys 20 us; by the ring 25; 32 of them 34 and 30).
//
// WIN_PARTS: otherwise; a workgroup per run of partitions, and a launch that joins them.
enum { WIN_WHOLE, WIN_FEW, WIN_PARTS };
constexpr int WIN_WHOLE_KEYS = 16000, WIN_SHORT_KEYS = 160;
static_assert(WIN_WHOLE_KEYS + HS_MAX_NODES + 4 * 32 <= 32 * WIN_RUN, "a walk's pages");
struct win_plan { int kind, part_keys, max_parts; };
win_plan plan_rows(const hs_ctx* ctx, int window, int sinks) {
    const long long cap = (long long)ctx->lim.max_blocks_per_seq * 16, nodes = 1 + ctx->lim.c_max * ctx->lim.k_max;
    const long long span = std::min<long long>(cap, window), s = std::min<long long>(cap, sinks);
    const long long units = (long long)ctx->lim.max_batch * ctx->desc.n_kv_heads;
    auto most = [&](long long part) {
        return std::min((s + part - 1) / part + (span + nodes - 2) / part + 2, (cap + part - 1) / part);
    };
    const int kind = span + s <= (units >= ctx->n_cu ? WIN_WHOLE_KEYS : WIN_SHORT_KEYS) ? WIN_WHOLE
                     : rows_of(ctx) <= 32 && units * (span + s) <= 64ll * 4 * ctx->n_cu ? WIN_FEW : WIN_PARTS;
    // Long partitions mean fewer partial results, which are written into the middle of the key stream; short ones keep a small batch spread
    // over the chip: a wavefront or a workgroup each.
    long long part = kind == WIN_FEW ? 1024 : 2048;
    while (part > 64 && units * ((span + part - 1) / part) < (kind == WIN_FEW ? 1024 : 512)) part /= 2;
    while (part < ctx->att_part && most(part) > ctx->max_parts) part *= 2;      // (what the workspace holds)
    if (most(part) > ctx->max_parts) part = ctx->att_part;
    return {kind, (int)part, (int)most(part)};
}

win_args make_args(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, const void* q,
                   void* out, int window, int sinks) {
    const hs_model_desc& d = ctx->desc;
    const size_t at = (size_t)layer * cache->n_blocks * d.n_kv_heads * 16 * d.head_dim;
    win_args a = {};
    a.q = (const bf16_t*)q;
    a.kc = (const bf16_t*)cache->k + at;
    a.vc = (const bf16_t*)cache->v + at;
    a.seq_len = seq->seq_len;
    a.block_table = seq->block_table;
    a.row_off = step->row_off;
    a.row2seq = step->row2seq;
    a.pos = step->pos;
    a.anc_mask = step->anc_mask;
    a.out = (bf16_t*)out;
    a.part_o = reinterpret_cast<_Float16*>(ctx->ws + ctx->lay.part_o);
    a.part_ml = reinterpret_cast<float*>(ctx->ws + ctx->lay.part_ml);
    a.batch = seq->batch;
    a.max_blocks = ctx->lim.max_blocks_per_seq;
    a.n_blocks = cache->n_blocks;
    a.hq = d.n_q_heads;
    a.hkv = d.n_kv_heads;
    a.window = window;
    a.sinks = sinks;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)d.head_dim);
    const win_plan p = plan_rows(ctx, window, sinks);
    a.kind = p.kind;
    a.lag = rows_of(ctx) <= 32 ? 0.f : 8.f;
    a.part_keys = p.part_keys;
    a.max_parts = p.max_parts;
    a.part_rows = (size_t)ctx->lim.max_rows * d.n_q_heads;
    return a;
}

}  // namespace

void hs_launch_window_attention(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step,
                                const void* q, void* out, int window, int sinks, hipStream_t st) {
    win_args a = make_args(ctx, layer, cache, seq, step, q, out, window, sinks);
    const int most = rows_of(ctx);
    if (a.kind == WIN_FEW) {
        a.groups = (a.max_parts + 3) / 4;
        const dim3 grid((unsigned)(a.groups * a.hkv * a.batch));
        if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((window_rows<128>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((window_rows<64>), grid, dim3(256), 0, st, a);
        return;
    }
    // How many workgroups share the partitions of a (sequence, KV head): as many as make the fewest tiles one after the other, in
    // rounds of two workgroups per compute unit, of which each takes as long as WIN_START tiles until its first one is there.
    const int tile_groups = (most + 127) / 128;
    long long best = 0;
    if (a.kind == WIN_WHOLE) a.groups = 1;
    for (int groups = 1; a.kind != WIN_WHOLE && groups <= a.max_parts; groups++) {
        const int run = (a.max_parts + groups - 1) / groups * (a.part_keys / 32);
        if (run > WIN_RUN) continue;      // (one partition is at most 64 tiles)
        const long long rounds = ((long long)groups * a.hkv * a.batch + 2 * ctx->n_cu - 1) / (2 * ctx->n_cu);
        const long long cost = rounds * (WIN_START + run);
        if (a.groups == 0 || cost < best) { best = cost; a.groups = groups; }
    }
    const dim3 grid((unsigned)(a.groups * a.hkv * a.batch * tile_groups));
    if (ctx->desc.head_dim == 128) {
        if (a.kind == WIN_WHOLE) hipLaunchKernelGGL((window_rows_ring<128, true>), grid, dim3(256), 0, st, a, tile_groups);
        else hipLaunchKernelGGL((window_rows_ring<128, false>), grid, dim3(256), 0, st, a, tile_groups);
    } else {
        if (a.kind == WIN_WHOLE) hipLaunchKernelGGL((window_rows_ring<64, true>), grid, dim3(256), 0, st, a, tile_groups);
        else hipLaunchKernelGGL((window_rows_ring<64, false>), grid, dim3(256), 0, st, a, tile_groups);
    }
}

void hs_launch_window_merge(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, void* out,
                            int window, int sinks, hipStream_t st) {
    const win_args a = make_args(ctx, 0, cache, seq, step, nullptr, out, window, sinks);
    if (a.kind == WIN_WHOLE) return;
    const int per = 4 * 512 / ctx->desc.head_dim, sets = (a.hq + per - 1) / per;      // heads of a workgroup, workgroups of a row
    const dim3 grid(hs_row_grid(ctx, 256, sets), sets);
    const bool early = ctx->lim.max_rows <= HS_EARLY_ROWS;
    if (ctx->desc.head_dim == 128) {
        if (early) hipLaunchKernelGGL((window_merge<128, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((window_merge<128, false>), grid, dim3(256), 0, st, a);
    } else {
        if (early) hipLaunchKernelGGL((window_merge<64, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((window_merge<64, false>), grid, dim3(256), 0, st, a);
    }
}

void hs_launch_window_chunk(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const int32_t* len_plus1,
                            const hs_step* step, const void* q, void* out, int chunk, int window, int sinks, hipStream_t st) {
    win_args a = make_args(ctx, layer, cache, seq, step, q, out, window, sinks);
    a.seq_len = len_plus1;
    a.lag = 8.f;
    // (a grid has fewer than 2^24 workgroups of 256: where that is too few, they take several blocks of rows)
    const long long most = std::max<long long>(1, (1ll << 23) / ((long long)a.hkv * a.batch));
    const int nx = (int)std::min(most, ((long long)chunk * (a.hq / a.hkv) + 127) / 128);
    const dim3 grid((unsigned)(nx * a.hkv * a.batch));
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((window_chunk<128>), grid, dim3(256), 0, st, a, nx);
    else hipLaunchKernelGGL((window_chunk<64>), grid, dim3(256), 0, st, a, nx);
}
