// Attention for a batch whose sequences share prefixes: the responses to one prompt, whose block tables name the same pages for the prompt's
// tokens (hs_pages_fork).  A row's result is what hs_verify's attention defines; what differs is who reads the keys.
//
//   out[row, h] = sum_t softmax_t(q[row, h] . k[t, h / G] / sqrt(head_dim)) v[t, h / G]
//
// The keys of a group's prefix [0, P) are seen by all rows of all members, whose query rows are neighbours in memory: a workgroup takes up to 128 of
// them, of whatever sequences, through a run of these keys, with no mask.  A member's own keys [P, L + nn) are walked for its own rows as usual.  Both
// leave partial results, which a second launch joins (a sequence without a prefix whose keys are one walk writes its result itself).
// P is the group's prefix length, cut to what every member with rows has cached and to whole tiles of 32 keys; what is cut off is read
// by each member through its own table.
//
// With 16 responses of one token, 28 query and 4 KV heads, a key is multiplied with 112 query rows per KV head: prefixes are bound by the matrix unit
// and own keys by memory, and both kinds of workgroups are in one launch, so that the ones' products and the others' loads overlap.
//
// The order of a row's sums is that of its keys: 32-key tiles; the runs of a prefix, which depend on its length, the limits and the hints given with
// the prefixes; own keys in partitions at multiples of part_keys.  It does not depend on what other rows there are.
#include <algorithm>

#include "hs_attention_ring.h"
#include "hs_internal.h"

using namespace hs_ring;

namespace {

struct shr_args {
    const bf16_t *q, *kc, *vc;          // kc, vc: at the layer
    const int32_t *seq_len, *block_table, *row_off, *row2seq, *group_off, *prefix_len;
    const uint64_t* anc_mask;
    bf16_t* out;
    _Float16* part_o;
    float* part_ml;
    int32_t* parts;                     // [batch] partial results of a sequence's rows; -1: they have their results
    int batch, n_groups, max_blocks, n_blocks, hq, hkv, sinks, part_keys, max_parts;
    int splits, prefix_tiles, prefix_units;      // runs of a prefix; groups of four row tiles per run in the grid; workgroups for prefixes
    int runs, tiles;                             // workgroups per (sequence, KV head) that share its partitions, and groups of four row tiles
    bool whole;                                  // own keys are one partition
    size_t part_rows;
    float scale_log2, lag;
};

// (The walk's keys: those from k0 on, without a gap.)
struct shr_span {
    int L, total, first, sink_end;
    __device__ __forceinline__ int skip(int kb) const { return kb; }
};

// A group: its members, of which `leader` is the first that has rows, and its keys [0, P), in n_pre runs.
struct group_info { int b0, b1, leader, P, n_pre; };
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ group_info load_group(const shr_args& a, int g, int lane) {
    group_info r;
    r.b0 = max(a.group_off[g], 0);
    r.b1 = min(a.group_off[g + 1], a.batch);
    int shortest = INT32_MAX, leader = INT32_MAX;
    for (int b = r.b0 + lane; b < r.b1; b += 64) {
        const bool rows = a.row_off[b + 1] > a.row_off[b];
        if (rows) {
            shortest = min(shortest, a.seq_len[b] - 1);
            leader = min(leader, b);
        }
    }
    r.leader = wave_min(leader);
    shortest = wave_min(shortest);
    const int most = min(min(a.prefix_len[g], shortest), a.max_blocks * 16);
    r.P = r.leader == INT32_MAX || a.splits == 0 ? 0 : max(most, 0) & ~31;
    r.P = hs_uniform(r.P);
    r.leader = hs_uniform(r.leader);
    r.n_pre = min(a.splits, r.P >> 5);
    return r;
}
// The group of a sequence: the last one that begins with it or before it, if it holds it.
__device__ __forceinline__ group_info group_of(const shr_args& a, int b, int lane) {
    int n = 0;
    for (int i = lane; i <= a.n_groups; i += 64) n += __popcll(__ballot(a.group_off[i] <= b));
    // (lanes that have left the loop count for the others: the sum is the first lane's, which stays in it longest)
    n = hs_uniform(n);
    if (n < 1 || n > a.n_groups) return {b, b + 1, b, 0, 0};
    return load_group(a, n - 1, lane);
}

// A workgroup with up to four row tiles at a time: either a run of a group's prefix for rows of all members (the first prefix_units workgroups),
// or partitions of a sequence's own keys for its rows.
template <int HD>
__global__ __launch_bounds__(256, 2) void shared_rows(shr_args a) {
    __shared__ __attribute__((aligned(1024))) win_lds<HD> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int G = a.hq / a.hkv;
    const bool prefix = (int)blockIdx.x < a.prefix_units;
    int j, r0, R, b_table, tile0, tile_step, turn, k0, k_end, part_keys, c;
    bool direct = false;
    shr_span s = {0, 0, 0, 0};
    if (prefix) {
        const int per = a.n_groups * a.hkv * a.splits, unit = blockIdx.x % per;
        const int split = unit % a.splits, g = unit / a.splits / a.hkv;
        j = unit / a.splits % a.hkv;
        const group_info gr = load_group(a, g, lane);
        if (split >= gr.n_pre) return;
        r0 = a.row_off[gr.b0];
        R = (a.row_off[gr.b1] - r0) * G;
        b_table = gr.leader;
        tile0 = 4 * (blockIdx.x / per);
        tile_step = 4 * a.prefix_tiles;
        turn = 0;
        const int tiles = gr.P >> 5;
        k0 = 32 * (int)((long long)tiles * split / gr.n_pre);
        k_end = 32 * (int)((long long)tiles * (split + 1) / gr.n_pre);
        part_keys = INT32_MAX / 2;
        c = split;
        s.L = s.total = gr.P;
        a.lag = 8.f;
    } else {
        const int per = a.batch * a.hkv * a.runs, unit = (blockIdx.x - a.prefix_units) % per, first = (blockIdx.x - a.prefix_units) / per;
        const int run = unit % a.runs;
        j = unit / a.runs % a.hkv;
        const int b = unit / a.runs / a.hkv;
        r0 = a.row_off[b];
        const int nn = a.row_off[b + 1] - r0;
        if (nn <= 0) return;
        R = nn * G;
        const group_info gr = group_of(a, b, lane);
        s.L = min(a.seq_len[b] - 1, INT32_MAX - (1 << 25));      // (sums with L stay in 32 bits: there are at most 2^25 rows)
        s.total = s.L < 0 ? 0 : min(s.L + nn, a.max_blocks * 16);
        s.total = min(s.total, max(s.L, 0) + HS_MAX_NODES);       // (no row sees a slot beyond those of 64 nodes)
        part_keys = a.whole ? INT32_MAX / 2 : a.part_keys;
        const int f = gr.P / part_keys;
        const int n = min(s.total > gr.P ? (s.total + part_keys - 1) / part_keys - f : 0, a.max_parts - gr.n_pre);
        direct = a.whole && gr.n_pre == 0;
        if (threadIdx.x == 0 && run == 0 && j == 0 && first == 0) a.parts[b] = direct ? -1 : gr.n_pre + n;
        const int c0 = (int)((long long)n * run / a.runs), c1 = (int)((long long)n * (run + 1) / a.runs);
        if (!direct && c0 >= c1) return;
        b_table = b;
        tile0 = 4 * first;
        tile_step = 4 * a.tiles;
        turn = run + j + b;
        k0 = max(gr.P, (f + c0) * part_keys);
        k_end = n == 0 ? k0 : (int)min((long long)s.total, (long long)(f + c1) * part_keys);
        c = gr.n_pre + c0;
    }
    const int32_t* bt = a.block_table + (size_t)b_table * a.max_blocks;
    const int nrt = (R + 31) >> 5;
    const int c_first = c;
    for (int tg = tile0; tg < nrt; tg += tile_step) {
        const int rt = tg + ((wave - turn) & 3);      // (wavefronts with rows are not the same ones everywhere)
        row_tile<HD> t;
        load_query_tile<HD>(a.q, prefix ? nullptr : a.anc_mask, r0, rt, R, G, a.hq, j, half, l32, t.qf, t.anc);
        t.lo = 0;
        t.hi = s.L;
        begin_tile<HD>(t);
        asm volatile("" : "+v"(t.anc));      // (waited for here, not in the loop)
        c = c_first;
        ring_keys<HD, true>(a, s, bt, j, k0, k_end, part_keys, 0, s.L, t, rt >= nrt, lds, [&]() __attribute__((always_inline)) {
            if (!direct) {
                put_partial<HD>(a, t, r0, rt, R, G, j, c, lane);
                begin_tile<HD>(t);
                c++;
            }
        });
        if (direct) put_result<HD>(a, t, r0, rt, R, G, j, lane);
    }
}

// Joins the partial results of a row's query heads in their order: a wavefront takes 512 / HD heads of a row, a lane eight elements of one, eight partial
// results at a time.
template <int HD>
__global__ __launch_bounds__(256) void shared_merge(shr_args a) {
    constexpr int LANES = HD / 8, HEADS = 64 / LANES, AHEAD = 8;
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63, head = (blockIdx.y * 4 + (threadIdx.x >> 6)) * HEADS + lane / LANES;
    if ((blockIdx.y * 4 + (threadIdx.x >> 6)) * HEADS >= a.hq) return;
    for (int row = blockIdx.x; (size_t)row * a.hq < a.part_rows; row += gridDim.x) {
        if (row >= a.row_off[a.batch]) return;
        const int n = a.parts[a.row2seq[row]];
        if (n < 0) continue;
        const size_t prow = (size_t)row * a.hq + min(head, a.hq - 1);
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + prow;
        const _Float16* po = a.part_o + prow * HD + 8 * (lane % LANES);
        float top = -INFINITY, den = 0.f, acc[8];
#pragma unroll
        for (int i = 0; i < 8; i++) acc[i] = 0.f;
        for (int p0 = 0; p0 < n; p0 += AHEAD) {
            float2 x[AHEAD];
            f16x8 v[AHEAD];
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                const int at = min(p0 + p, n - 1);
                x[p] = ml[at * a.part_rows];
                v[p] = *reinterpret_cast<const f16x8*>(po + at * a.part_rows * HD);
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
                const float w = fast_exp2(x[p].x - safe) * x[p].y;      // (the partial result is stored normalised)
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

// How keys are cut and shared out: a function of the limits and of the hints that come with the prefixes (not of a step's rows), since the order of
// a row's sums follows from it; and, from what rows to expect, how many workgroups a launch has.
constexpr int SHARED_WHOLE_KEYS = 16000, SHARED_SHORT_KEYS = 160;
struct shr_plan { int part_keys, max_parts, splits; bool whole; };
shr_plan plan_keys(const hs_ctx* ctx, const hs_shared_prefix* pre) {
    const hs_limits& l = ctx->lim;
    const hs_model_desc& d = ctx->desc;
    const long long cap = (long long)l.max_blocks_per_seq * 16, longest = std::min<long long>(pre->max_prefix, cap);
    const long long span = std::max<long long>(cap - longest, 32), G = d.n_q_heads / d.n_kv_heads;
    const long long rows = G * pre->max_members * (1 + l.c_max * l.k_max);
    shr_plan p;
    // runs of a prefix: two workgroups per compute unit with 128 rows each, of 256 keys at least
    const long long units = (long long)pre->n_groups * d.n_kv_heads * ((rows + 127) / 128);
    long long splits = std::max(1ll, std::min(longest / 256, (2 * ctx->n_cu + units - 1) / units));
    splits = std::min(splits, 32ll);
    if (longest < 32) splits = 0;
    const long long pairs = (long long)l.max_batch * d.n_kv_heads;
    p.whole = span <= (pairs >= ctx->n_cu ? SHARED_WHOLE_KEYS : SHARED_SHORT_KEYS);
    // (one partition more than keys are cut into: the one that a prefix ends in)
    long long part = 2048;
    while (part > 128 && pairs * ((span + part - 1) / part) < 4ll * ctx->n_cu) part /= 2;
    auto own = [&](long long n) { return p.whole ? 1ll : (cap + n - 1) / n; };
    while (own(part) + 1 > ctx->max_parts && part < cap) part *= 2;
    splits = std::min(splits, ctx->max_parts - own(part));
    p.splits = (int)std::max(0ll, splits);
    p.part_keys = (int)part;
    p.max_parts = std::max(ctx->max_parts, 1);
    return p;
}

shr_args make_args(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, const hs_shared_prefix* pre,
                   const void* q, void* out) {
    const hs_model_desc& d = ctx->desc;
    const size_t at = (size_t)layer * cache->n_blocks * d.n_kv_heads * 16 * d.head_dim;
    shr_args a = {};
    a.q = (const bf16_t*)q;
    a.kc = (const bf16_t*)cache->k + at;
    a.vc = (const bf16_t*)cache->v + at;
    a.seq_len = seq->seq_len;
    a.block_table = seq->block_table;
    a.row_off = step->row_off;
    a.row2seq = step->row2seq;
    a.anc_mask = step->anc_mask;
    a.group_off = pre->group_off;
    a.prefix_len = pre->prefix_len;
    a.n_groups = pre->n_groups;
    a.out = (bf16_t*)out;
    a.part_o = reinterpret_cast<_Float16*>(ctx->ws + ctx->lay.part_o);
    a.part_ml = reinterpret_cast<float*>(ctx->ws + ctx->lay.part_ml);
    a.parts = reinterpret_cast<int32_t*>(ctx->ws + ctx->lay.shared_parts);
    a.batch = seq->batch;
    a.max_blocks = ctx->lim.max_blocks_per_seq;
    a.n_blocks = cache->n_blocks;
    a.hq = d.n_q_heads;
    a.hkv = d.n_kv_heads;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)d.head_dim);
    a.part_rows = (size_t)ctx->lim.max_rows * d.n_q_heads;
    const shr_plan p = plan_keys(ctx, pre);
    a.part_keys = p.part_keys;
    a.max_parts = p.max_parts;
    a.splits = p.splits;
    a.whole = p.whole;
    const int G = d.n_q_heads / d.n_kv_heads, nodes = 1 + ctx->lim.c_max * ctx->lim.k_max;
    a.lag = G * nodes <= 32 ? 0.f : 8.f;
    // row tiles in the grid: of a group by the rows that are expected, if anything is known of them; a workgroup takes further ones in turn
    const long long most = (long long)pre->max_members * nodes;
    const long long expect = step->rows_hint > 0 ? std::min<long long>(most, 5ll * step->rows_hint / (4 * pre->n_groups) + 1) : most;
    const long long run_units = std::max(1ll, (long long)a.n_groups * a.hkv * a.splits);
    a.prefix_tiles = (int)std::max<long long>(1, std::min((expect * G + 127) / 128, (1ll << 20) / run_units));
    a.tiles = (G * nodes + 127) / 128;
    a.runs = 1;
    if (!a.whole) {
        const long long cap = (long long)a.max_blocks * 16, own = (cap + a.part_keys - 1) / a.part_keys, pairs = (long long)a.batch * a.hkv;
        a.runs = (int)std::max(1ll, std::min(own, (8ll * ctx->n_cu + pairs - 1) / pairs));
    }
    a.prefix_units = a.n_groups * a.hkv * a.splits * a.prefix_tiles;
    return a;
}

}  // namespace

void hs_launch_shared_attention(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step,
                                const hs_shared_prefix* pre, const void* q, void* out, hipStream_t st) {
    const shr_args a = make_args(ctx, layer, cache, seq, step, pre, q, out);
    const dim3 grid((unsigned)(a.prefix_units + a.batch * a.hkv * a.runs * a.tiles));
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((shared_rows<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((shared_rows<64>), grid, dim3(256), 0, st, a);
}

void hs_launch_shared_merge(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, const hs_shared_prefix* pre,
                            void* out, hipStream_t st) {
    const shr_args a = make_args(ctx, 0, cache, seq, step, pre, nullptr, out);
    const int per = 4 * 512 / ctx->desc.head_dim, sets = (a.hq + per - 1) / per;      // heads of a workgroup, workgroups of a row
    const dim3 grid(hs_row_grid(ctx, 256, sets), sets);
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((shared_merge<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((shared_merge<64>), grid, dim3(256), 0, st, a);
}
