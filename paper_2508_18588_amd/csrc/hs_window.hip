// Paged attention with a sliding window and sinks: a query row at position p sees, of the keys that it would see without
// a window (the cached ones and its ancestors among the draft's nodes, or the tokens of its chunk up to itself), those at
// positions t > p - window and those at t < sinks.
//
//   out[row, h] = sum_t softmax_t(q[row, h] . k[t, h / G] / sqrt(head_dim)) v[t, h / G]  over the visible t; 0 if there is none
//
// A sequence of L cached tokens and nn rows needs the keys [0, sinks) and [L + 1 - window, L + nn), whatever its length: only
// their pages are looked up and read.
//
// One wavefront takes a tile of 32 query rows (rows of one token's G query heads, which share a KV head, are neighbours) through
// a run of keys, 32 at a time, without the LDS: the matrix instructions' operands are loaded from the cache as they are needed.
// Scores are computed transposed, S^T = K . Q^T (v_mfma_f32_32x32x16_bf16), so that a lane has the scores of one query row and the
// softmax statistics are its own scalars.  The second product O^T = V^T . P^T takes 16 tokens of V^T, which the cache holds token
// index fastest: a lane's operand is 16 contiguous bytes, tokens 8 half .. 8 half + 7 of a page.  The rows of the first product's
// operand are therefore the page's keys in the order of page_order, which leaves a lane exactly the probabilities of those tokens.
//
// Every sum has an order that depends on absolute key positions only (32-key tiles, partitions of part_keys, merged in index order;
// keys that a row does not see contribute exact zeros): a row's result does not depend on what other rows are computed with it.
#include <algorithm>

#include "hs_attention_tile.h"
#include "hs_internal.h"

namespace {

struct win_args {
    const bf16_t *q, *kc, *vc;          // kc, vc: at the layer
    const int32_t *seq_len, *block_table, *row_off, *row2seq, *pos;
    const uint64_t* anc_mask;
    bf16_t* out;
    _Float16* part_o;
    float* part_ml;
    int batch, max_blocks, n_blocks, hq, hkv, window, sinks, part_keys, max_parts;
    float scale_log2;
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
    s.L = min(seq_len - 1, cap);
    s.total = min(s.L + nn, cap);
    s.first = max(0, s.L + 1 - a.window);
    s.sink_end = min(min(a.sinks, s.first), s.total);
    s.n_sink = (s.sink_end + a.part_keys - 1) / a.part_keys;
    s.p_first = max(s.first / a.part_keys, s.n_sink);
    // (no more than there is room for: a draft of more nodes than the limits allow is not laid out by anybody)
    s.n_parts = s.L < 0 || nn <= 0 ? 0 : min(a.max_parts, s.n_sink + max(0, (s.total + a.part_keys - 1) / a.part_keys - s.p_first));
    return s;
}

// What a lane's query row sees: keys below hi that lie from lo on or below `sinks`, and of the slots from L on the nodes of anc.
template <int HD>
struct row_tile {
    bf16x8 qf[HD / 16];
    f32x16 o[HD / 32];
    float m, l;
    int lo, hi;
    uint64_t anc;
};

// A page's key that is row r of the first product's operand (its own inverse): the result's rows 8 a + 4 h + c, of which a lane of
// half h has those of its h, are keys 8 h + 4 a + c.
__device__ __forceinline__ int page_order(int r) { return (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1); }

template <int HD>
struct key_tile { bf16x8 k[HD / 16]; };
template <int HD>
struct value_tile { bf16x8 v[2][HD / 32]; };

__device__ __forceinline__ bool has_nonfinite(const bf16x8& x) {
    const u32x4 u = __builtin_bit_cast(u32x4, x);
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; i++) any |= (u[i] & 0x7F80u) == 0x7F80u || (u[i] & 0x7F800000u) == 0x7F800000u;
    return any;
}

// Walks keys k0, ... (32 at a time, k_end excluded) with one row tile.  all_lo, all_hi: every row sees the keys in [all_lo, all_hi) and
// in [0, min(sinks, all_hi)).
template <int HD>
__device__ __forceinline__ void walk_keys(const win_args& a, const win_span& s, const int32_t* __restrict__ bt, int j, int k0, int k_end,
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
    struct places { int p0, p1; };
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
            for (int dt = 0; dt < NDT; dt++) v.v[pp][dt] = *reinterpret_cast<const bf16x8*>(src + dt * 32 * 16);
        }
    };

    if (k0 >= k_end) return;
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
        const bool masked = kb + 32 > all_hi || !(kb >= all_lo || kb + 32 <= a.sinks) || here.p0 < 0 || here.p1 < 0;
        unsigned seen = 0xFFFFu;        // bit e: the row sees key e of the lane's
        if (masked) {
            seen = 0;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const int key = kb + 16 * (e >> 3) + 8 * half + (e & 7);
                const bool old = key < t.hi && (key >= t.lo || key < a.sinks);
                const bool node = key >= s.L && key - s.L < 64 && ((t.anc >> ((key - s.L) & 63)) & 1ull);
                const bool vis = (old || node) && (e < 8 ? here.p0 : here.p1) >= 0;
                sc[e] = vis ? sc[e] : -INFINITY;
                seen |= (unsigned)vis << e;
            }
        }
        float tmax = sc[0];
#pragma unroll
        for (int e = 1; e < 16; e++) tmax = fmaxf(tmax, sc[e]);
        {
            // lanes l and l + 32 hold the two halves of a query row
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(tmax), __float_as_uint(tmax), false, false);
            tmax = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale_log2;
        }
        const float m_new = fmaxf(t.m, tmax);
        float alpha = 1.f;
        if (__any(m_new != t.m)) {
            alpha = fast_exp2(t.m - (m_new == -INFINITY ? 0.f : m_new));
            t.m = m_new;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
#pragma unroll
                for (int e = 0; e < 16; e++) t.o[dt][e] *= alpha;
        }
        const float m_safe = t.m == -INFINITY ? 0.f : t.m;
        float psum = 0.f;
        bf16x8 pb[2];
#pragma unroll
        for (int e = 0; e < 16; e++) {
            // (probabilities are rounded to bf16, the matrix instruction's type: half a step, 2^-9, each; their sum is not)
            const float p = fast_exp2(__builtin_fmaf(sc[e], a.scale_log2, -m_safe));
            psum += p;
            pb[e >> 3][e & 7] = (__bf16)p;
        }
        {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(psum), __float_as_uint(psum), false, false);
            t.l = __builtin_fmaf(t.l, alpha, __uint_as_float(sw[0]) + __uint_as_float(sw[1]));
        }
        bool odd = false;
        if (masked) {
#pragma unroll
            for (int pp = 0; pp < 2; pp++)
#pragma unroll
                for (int dt = 0; dt < NDT; dt++) odd |= has_nonfinite(v.v[pp][dt]);
        }
        if (!__any(odd)) {
#pragma unroll
            for (int pp = 0; pp < 2; pp++)
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    t.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v[pp][dt], pb[pp], t.o[dt], 0, 0, 0);
        } else {
            // An infinity or a NaN among the values of a tile that not every row sees all of: 0 times that is a NaN.  Token by
            // token, and a row that does not see the token keeps what it had.
#pragma unroll 1
            for (int th = 0; th < 16; th++) {
                const int th_half = th >> 3, th_at = th & 7;
#pragma unroll
                for (int pp = 0; pp < 2; pp++) {
                    const unsigned bits = __shfl((int)seen, l32 + 32 * th_half);
                    const bool sees = (bits >> (8 * pp + th_at)) & 1u;
#pragma unroll
                    for (int dt = 0; dt < NDT; dt++) {
                        bf16x8 one;
#pragma unroll
                        for (int e = 0; e < 8; e++) one[e] = half == th_half && e == th_at ? v.v[pp][dt][e] : (__bf16)0.f;
                        const f32x16 with = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, pb[pp], t.o[dt], 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; e++) t.o[dt][e] = sees ? with[e] : t.o[dt][e];
                    }
                }
            }
        }
        if (!more) return;
        load_v(cur, v);
        kb = next;
    }
}

// The rows of a draft (any number of nodes, a single token among them).  A workgroup takes four partitions of one (sequence, KV head)
// with all row tiles: its wavefronts take (partition, row tile) pairs in turn, neighbours share a partition's keys.
template <int HD>
__global__ __launch_bounds__(256, 2) void window_rows(win_args a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
    const int groups = (a.max_parts + 3) / 4;
    const int g = blockIdx.x % groups, pair = blockIdx.x / groups;
    const int j = pair % a.hkv, b = pair / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0;
    const win_span s = make_span(a.seq_len[b], nn, a);
    if (4 * g >= s.n_parts) return;
    const int G = a.hq / a.hkv, R = nn * G, nrt = (R + 31) >> 5;
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    const int items = min(4, s.n_parts - 4 * g) * nrt;
    for (int it = wave; it < items; it += 4) {
        const int c = 4 * g + it / nrt, rt = it % nrt;
        row_tile<HD> t;
        load_query_tile<HD>(a.q, a.anc_mask, r0, rt, R, G, a.hq, j, half, l32, t.qf, t.anc);
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
            for (int e = 0; e < 16; e++) t.o[dt][e] = 0.f;
        t.m = -INFINITY;
        t.l = 0.f;
        // the row's window; its depth is below nn, so that from all_lo on every row sees every cached key
        const int all_lo = max(0, s.L + nn - a.window), rho = rt * 32 + l32;
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
        const int p = s.partition(c);
        walk_keys<HD>(a, s, bt, j, s.skip(p * a.part_keys), min(s.total, (p + 1) * a.part_keys), all_lo, s.L, t, lane);
        store_partial<HD>(t.o, t.m, t.l, a.part_o, a.part_ml, r0, rt, R, G, a.hq, j, a.max_parts, c, half, l32);
    }
}

// Joins the partitions of one (row, query head) in their order: one wavefront each, four per workgroup.
template <int HD>
__global__ __launch_bounds__(256) void window_merge(win_args a) {
    constexpr int E = HD / 64;
    typedef _Float16 piece __attribute__((ext_vector_type(E)));
    const int head = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (head >= a.hq) return;
    const int M = a.row_off[a.batch];
    for (int row = blockIdx.x; row < M; row += gridDim.x) {
        const int b = a.row2seq[row];
        const int n = make_span(a.seq_len[b], a.row_off[b + 1] - a.row_off[b], a).n_parts;
        const size_t prow = ((size_t)row * a.hq + head) * a.max_parts;
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + prow;
        const _Float16* po = a.part_o + prow * HD + E * lane;
        float top = -INFINITY;
        for (int p = lane; p < n; p += 64) top = fmaxf(top, ml[p].x);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        float den = 0.f, acc[E];
#pragma unroll
        for (int i = 0; i < E; i++) acc[i] = 0.f;
        for (int p = 0; p < n; p++) {
            const float2 x = ml[p];
            // the partition's weight in the whole; its output is stored normalised
            const float w = x.x == -INFINITY ? 0.f * x.y : fast_exp2(x.x - top) * x.y;
            const piece v = *reinterpret_cast<const piece*>(po + (size_t)p * HD);
            den += w;
#pragma unroll
            for (int i = 0; i < E; i++) acc[i] += w * (float)v[i];
        }
        bf16_t* dst = a.out + ((size_t)row * a.hq + head) * HD + E * lane;
#pragma unroll
        for (int i = 0; i < E; i++) dst[i] = f32_to_bf16(den == 0.f ? 0.f : acc[i] / den);
    }
}

// The rows of a chunk: consecutive tokens, row i of a sequence at position L + i.  A workgroup takes 128 query rows of one (sequence, KV
// head), a wavefront 32 of them through all their keys: with hundreds of rows per sequence there is enough to do without cutting the
// key axis.
template <int HD>
__global__ __launch_bounds__(256, 2) void window_chunk(win_args a, int nx) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
    const int pair = blockIdx.x / nx, j = pair % a.hkv, b = pair / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0;
    const win_span s = make_span(a.seq_len[b], nn, a);
    if (s.n_parts == 0) return;
    const int G = a.hq / a.hkv, R = nn * G;
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    for (int rt = (blockIdx.x % nx) * 4 + wave; rt * 32 < R; rt += nx * 4) {
        row_tile<HD> t;
        load_query_tile<HD>(a.q, nullptr, r0, rt, R, G, a.hq, j, half, l32, t.qf, t.anc);
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
            for (int e = 0; e < 16; e++) t.o[dt][e] = 0.f;
        t.m = -INFINITY;
        t.l = 0.f;
        const int rho = rt * 32 + l32;
        const int node0 = rt * 32 / G, node1 = min(nn - 1, (rt * 32 + 31) / G), node = min(rho / G, nn - 1);
        t.lo = max(0, s.L + node + 1 - a.window);
        t.hi = s.L + node + 1;
        win_span w = s;     // the keys of this tile's rows
        w.first = max(0, s.L + node0 + 1 - a.window);
        w.sink_end = min(min(a.sinks, w.first), s.total);
        walk_keys<HD>(a, w, bt, j, w.skip(0), min(s.total, s.L + node1 + 1), max(0, s.L + node1 + 1 - a.window), s.L + node0 + 1, t,
                      lane);
        if (rho >= R) continue;
        const float inv = t.l == 0.f ? 0.f : 1.f / t.l;
        bf16_t* po = a.out + ((size_t)(r0 + node) * a.hq + j * G + (rho - node * G)) * HD;
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
            for (int g4 = 0; g4 < 4; g4++) {
                u32x2 x;
                x.x = (uint32_t)f32_to_bf16(t.o[dt][4 * g4] * inv) | ((uint32_t)f32_to_bf16(t.o[dt][4 * g4 + 1] * inv) << 16);
                x.y = (uint32_t)f32_to_bf16(t.o[dt][4 * g4 + 2] * inv) | ((uint32_t)f32_to_bf16(t.o[dt][4 * g4 + 3] * inv) << 16);
                *reinterpret_cast<u32x2*>(po + dt * 32 + 8 * g4 + 4 * half) = x;
            }
    }
}

// Partitions of a draft's keys: their length, and the most that a sequence can have.  A function of the context's limits, the window
// and the sinks, so that the order of a row's sums is the same in every step.
struct win_plan { int part_keys, max_parts; };
win_plan plan_rows(const hs_ctx* ctx, int window, int sinks) {
    const long long cap = (long long)ctx->lim.max_blocks_per_seq * 16, nodes = 1 + ctx->lim.c_max * ctx->lim.k_max;
    const long long span = std::min<long long>(cap, window), s = std::min<long long>(cap, sinks);
    auto most = [&](long long part) {
        return std::min((s + part - 1) / part + (span + nodes - 2) / part + 2, (cap + part - 1) / part);
    };
    long long part = 1024;
    while (part > 64 && (long long)ctx->lim.max_batch * ctx->desc.n_kv_heads * ((span + part - 1) / part) < 2048) part /= 2;
    while (part < ctx->att_part && most(part) > ctx->max_parts) part *= 2;      // (what the workspace holds)
    if (most(part) > ctx->max_parts) part = ctx->att_part;
    return {(int)part, (int)most(part)};
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
    a.part_keys = p.part_keys;
    a.max_parts = p.max_parts;
    return a;
}

}  // namespace

void hs_launch_window_attention(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step,
                                const void* q, void* out, int window, int sinks, hipStream_t st) {
    const win_args a = make_args(ctx, layer, cache, seq, step, q, out, window, sinks);
    const dim3 grid((unsigned)((a.max_parts + 3) / 4 * a.hkv * a.batch));
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((window_rows<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((window_rows<64>), grid, dim3(256), 0, st, a);
}

void hs_launch_window_merge(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, void* out,
                            int window, int sinks, hipStream_t st) {
    const win_args a = make_args(ctx, 0, cache, seq, step, nullptr, out, window, sinks);
    const dim3 grid(hs_row_grid(ctx, 256, (a.hq + 3) / 4), (a.hq + 3) / 4);
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((window_merge<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((window_merge<64>), grid, dim3(256), 0, st, a);
}

void hs_launch_window_chunk(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const int32_t* len_plus1,
                            const hs_step* step, const void* q, void* out, int chunk, int window, int sinks, hipStream_t st) {
    win_args a = make_args(ctx, layer, cache, seq, step, q, out, window, sinks);
    a.seq_len = len_plus1;
    const int nx = (int)(((long long)chunk * (a.hq / a.hkv) + 127) / 128);
    const dim3 grid((unsigned)(nx * a.hkv * a.batch));
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((window_chunk<128>), grid, dim3(256), 0, st, a, nx);
    else hipLaunchKernelGGL((window_chunk<64>), grid, dim3(256), 0, st, a, nx);
}
