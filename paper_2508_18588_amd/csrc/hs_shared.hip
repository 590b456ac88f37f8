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
// and own keys by memory, and both kinds of workgroups are in one launch, so that the ones' products and the others' loads overlap.  Times here
// are those of both launches.  16 prompts of 1500 to 4500 tokens, 16 sequences each with drafts and up to 2048 own tokens, 4 KV heads: prefixes alone
// 108 us, own keys alone 114 (4.2 TB/s), together 160; 64 trees of 17 nodes behind 8000 tokens, 40 and 8 heads: 205 us, nearly all of them the prefix
// (880 TFLOP/s; the matrix unit is busy 47 % of the time, the vector unit 53 %, LDS 24 %, two wavefronts per SIMD to overlap them).
//
// The order of a row's sums is that of its keys: 32-key tiles; the runs of a prefix, which depend on its length, the limits and the hints given with
// the prefixes; own keys in partitions at multiples of part_keys.  It does not depend on what other rows there are, but through P where a member has not
// cached the group's whole prefix.
#include <algorithm>

#include "hs_attention_ring.h"
#include "hs_internal.h"
#include "hs_lanes.h"

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
    int own_units;                               // ... and in front of them those for own keys
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
    v = min(v, (int)lane_xor<32>((unsigned)v));
    v = min(v, (int)lane_xor<16>((unsigned)v));
    v = min(v, (int)lane_xor<8>((unsigned)v));
    v = min(v, (int)lane_xor<4>((unsigned)v));
    v = min(v, (int)lane_xor<2>((unsigned)v));
    return min(v, (int)lane_xor<1>((unsigned)v));
}
__device__ __forceinline__ group_info load_group(const shr_args& a, int g, int lane) {
    group_info r;
    r.b0 = max(a.group_off[g], 0);
    r.b1 = min(a.group_off[g + 1], a.batch);
    int shortest = INT32_MAX, leader = INT32_MAX;
    const int length = a.prefix_len[g];
    for (int b = r.b0 + lane; b < r.b1; b += 64) {
        const bool rows = a.row_off[b + 1] > a.row_off[b];
        if (rows) {
            shortest = min(shortest, a.seq_len[b] - 1);
            leader = min(leader, b);
        }
    }
    r.leader = wave_min(leader);
    shortest = wave_min(shortest);
    const int most = min(min(length, shortest), a.max_blocks * 16);
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

// As load_pair, but the caches may keep what is loaded: other workgroups read the same keys for other rows.
__device__ __forceinline__ __attribute__((always_inline)) void load_pair_kept(const unsigned char* base, unsigned off0, unsigned off1, unsigned lds_off,
                                                                              const int add) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3 offset:%4\n\tglobal_load_lds_dwordx4 %2, %3 offset:%5"
                 :
                 : "s"(lds_off), "v"(off0), "v"(off1), "s"(base), "i"(add), "i"(add + 1024)
                 : "memory", "m0");
}

// Tiles first, ... of a prefix with a row tile per wavefront, all of whose rows see all keys.  Key tiles come two at a time through the halves of the
// ring: one half is multiplied while the other one is filled.  There is a barrier for two tiles and not for each, between which wavefronts drift
// apart, so that of the two of a SIMD one has products for the matrix unit while the other one computes weights.  (With a barrier for each, as in
// ring_keys, the trees took 249 us; so 216, and 208 since wavefronts with products go first and nothing of own_rows is live here.)  idle: the wavefront has no rows,
// only its share of the tiles.  page: room for the numbers of 2 STEP_RUN pages.
constexpr int STEP_RUN = WIN_RUN;
template <int HD>
__device__ __forceinline__ void step_keys(const shr_args& a, const int32_t* __restrict__ bt, int j, int first, int n_tiles, row_tile<HD>& t, bool idle,
                                          unsigned char* ring, int* page_of) {
    using T = sub_tile<HD>;
    constexpr int NKS = HD / 16, NDT = HD / 32, CPW = T::PAGE / 1024, STEP = WIN_RING / 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    // the wavefront's share of a step: both pages' K (is_v = 0) or V^T of a tile
    const unsigned page_bytes = (unsigned)a.hkv * T::PAGE;
    const int is_v = wave & 1, my_tile = wave >> 1;
    const unsigned ring_off = (unsigned)(size_t)(hs_gemm_detail::lds_ptr_t)ring + my_tile * T::BYTES + is_v * T::V;
    const unsigned char* base = reinterpret_cast<const unsigned char*>(is_v ? a.vc : a.kc) + (size_t)j * T::PAGE;
    const unsigned from = is_v ? T::v_from(lane) : T::k_at(lane / (HD / 8), lane % (HD / 8));
    const int key_row = (l32 & 16) | page_order(l32 & 15);
    for (int u0 = 0; u0 < n_tiles; u0 += STEP_RUN) {
        const int n = min(n_tiles - u0, STEP_RUN);
        __syncthreads();      // (the ring and the pages have been read)
        bool missing = false;
        for (int i = tid; i < 2 * n; i += 256) {
            const int page = bt[2 * (first + u0) + i];
            page_of[i] = page < a.n_blocks ? page : -1;
            missing |= page < 0 || page >= a.n_blocks;
        }
        const bool holes = __syncthreads_or(missing);
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) asm volatile("" : "+v"(t.qf[ks]));      // (waited for here, see ring_keys)
        auto fetch = [&](int at, int buf) __attribute__((always_inline)) {      // the step that begins with tile at
            if (at + my_tile >= n) return;
#pragma unroll
            for (int pg = 0; pg < 2; pg++) {
                const int page = max(__builtin_amdgcn_readfirstlane(page_of[2 * (at + my_tile) + pg]), 0);
                const unsigned char* src = base + (size_t)page * page_bytes;
                const unsigned dst = ring_off + buf * STEP * T::BYTES + pg * T::PAGE;
#pragma unroll
                for (int i = 0; i < CPW; i += 2) load_pair_kept(src, is_v ? from : from ^ T::k_step(i), is_v ? from : from ^ T::k_step(i + 1), dst, i * 1024);
            }
        };
        fetch(0, 0);
        for (int at = 0, buf = 0; at < n; at += STEP, buf ^= 1) {
            // this step has landed (every wavefront has waited for its share), and the one before has been read
            HS_WAIT_VMCNT(0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            fetch(at + STEP, buf ^ 1);
            if (idle) continue;
            const unsigned char* step = ring + buf * STEP * T::BYTES;
            auto scores = [&](int x) __attribute__((always_inline)) {
                key_tile<HD> k;
                int k_at = T::k_at(key_row, half);
                asm volatile("" : "+v"(k_at));
#pragma unroll
                for (int ks = 0; ks < NKS; ks++) k.k[ks] = *reinterpret_cast<const bf16x8*>(step + x * T::BYTES + (k_at ^ (ks << 5)));
                f32x16 sc;
#pragma unroll
                for (int e = 0; e < 16; e++) sc[e] = 0.f;
#pragma unroll
                for (int ks = 0; ks < NKS; ks++) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.k[ks], t.qf[ks], sc, 0, 0, 0);
                return sc;
            };
            // (the next tile's first product needs nothing of this one's weights)
            auto tile = [&](int x, f32x16& sc, f32x16& next) __attribute__((always_inline)) {
                value_tile<HD> v;
#pragma unroll
                for (int pp = 0; pp < 2; pp++)
#pragma unroll
                    for (int dt = 0; dt < NDT; dt++)
                        v.v[pp][dt] = *reinterpret_cast<const bf16x8*>(step + x * T::BYTES + T::V + pp * T::PAGE + dt * 1024 + T::v_at(l32, half));
                if (holes) {      // pages that there are none of: their keys are not seen
                    const int p0 = __builtin_amdgcn_readfirstlane(page_of[2 * (at + x)]), p1 = __builtin_amdgcn_readfirstlane(page_of[2 * (at + x) + 1]);
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if ((e < 8 ? p0 : p1) < 0) sc[e] = -INFINITY;
#pragma unroll
                    for (int pp = 0; pp < 2; pp++)
#pragma unroll
                        for (int dt = 0; dt < NDT; dt++)
                            if ((pp ? p1 : p0) < 0) v.v[pp][dt] = {};
                }
                const float alpha = take_scores<HD>(a, shr_span{}, t, sc, places{}, false, 0, half);
                __builtin_amdgcn_s_setprio(1);
                if (x + 1 < STEP) next = scores(x + 1);      // (beyond the run: of whatever lies there, not used)
                bf16x8 pb[2];
                take_probabilities<HD>(a, t, sc, alpha, pb);
                take_values<HD>(t, v, pb);
                __builtin_amdgcn_s_setprio(0);
            };
            f32x16 even = scores(0), odd;
            tile(0, even, odd);
            if (at + 1 < n) tile(1, odd, odd);
        }
    }
}

// A run of a group's prefix for rows of all members, four row tiles at a time.
template <int HD>
__device__ __forceinline__ void prefix_rows(const shr_args& args, win_lds<HD>& lds) {
    shr_args a = args;
    a.lag = 8.f;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Eight runs at a time for all their rows: those that read the same keys have ids eight apart, on one XCD, and begin together, so that its L2 has them
    // for all (256 sequences with drafts, eight workgroups a run: 164 us; with a run's workgroups 192 ids apart 169).
    const int G = a.hq / a.hkv, at = blockIdx.x - a.own_units, unit = at / (8 * a.prefix_tiles) * 8 + at % 8, first_tile = 4 * (at / 8 % a.prefix_tiles);
    if (unit >= a.n_groups * a.hkv * a.splits) return;
    const int split = unit % a.splits, g = unit / a.splits / a.hkv, j = unit / a.splits % a.hkv;
    const group_info gr = load_group(a, g, lane);
    if (split >= gr.n_pre) return;
    const int r0 = a.row_off[gr.b0], R = (a.row_off[gr.b1] - r0) * G, nrt = (R + 31) >> 5, tiles = gr.P >> 5;
    const int first = (int)((long long)tiles * split / gr.n_pre), end = (int)((long long)tiles * (split + 1) / gr.n_pre);
    const int32_t* bt = a.block_table + (size_t)gr.leader * a.max_blocks;
    for (int tg = first_tile; tg < nrt; tg += 4 * a.prefix_tiles) {
        const int rt = tg + wave;
        row_tile<HD> t;
        load_query_tile<HD>(a.q, nullptr, r0, rt, R, G, a.hq, j, lane >> 5, lane & 31, t.qf, t.anc);
        begin_tile<HD>(t);
        step_keys<HD>(a, bt, j, first, end - first, t, rt >= nrt, lds.ring, lds.page);
        put_partial<HD>(a, t, r0, rt, R, G, j, split, lane);
    }
}

// Partitions of a sequence's own keys for its rows.
template <int HD>
__device__ __forceinline__ void own_rows(const shr_args& a, win_lds<HD>& lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = a.batch * a.hkv * a.runs, unit = blockIdx.x % per, first = blockIdx.x / per;
    const int pair = unit / a.runs, run = (unit + (pair >> 3)) % a.runs;      // (ids are dealt to eight XCDs in turn: none gets the same run of all)
    const int j = pair % a.hkv, b = pair / a.hkv, G = a.hq / a.hkv;
    const int r0 = a.row_off[b], nn = a.row_off[b + 1] - r0, R = nn * G, nrt = (R + 31) >> 5;
    shr_span s = {0, 0, 0, 0};
    s.L = min(a.seq_len[b] - 1, INT32_MAX - (1 << 25));      // (sums with L stay in 32 bits: there are at most 2^25 rows)
    const group_info gr = group_of(a, b, lane);              // (asked for before it is known whether there are rows: one trip to memory)
    if (nn <= 0) return;
    s.total = s.L < 0 ? 0 : min(s.L + nn, a.max_blocks * 16);
    s.total = min(s.total, max(s.L, 0) + HS_MAX_NODES);       // (no row sees a slot beyond those of 64 nodes)
    const int part_keys = a.whole ? INT32_MAX / 2 : a.part_keys, f = gr.P / part_keys;
    const int n = min(s.total > gr.P ? (s.total - 1) / part_keys + 1 - f : 0, a.max_parts - gr.n_pre);
    const bool direct = a.whole && gr.n_pre == 0;
    if (threadIdx.x == 0 && run == 0 && j == 0 && first == 0) a.parts[b] = direct ? -1 : gr.n_pre + n;
    const int c0 = (int)((long long)n * run / a.runs), c1 = (int)((long long)n * (run + 1) / a.runs);
    if (!direct && c0 >= c1) return;
    const int k0 = max(gr.P, (f + c0) * part_keys);
    const int k_end = n == 0 ? k0 : (int)min((long long)s.total, (long long)(f + c1) * part_keys);
    const int32_t* bt = a.block_table + (size_t)b * a.max_blocks;
    for (int tg = 4 * first; tg < nrt; tg += 4 * a.tiles) {
        const int rt = tg + ((wave - (run + j + b)) & 3);      // (wavefronts with rows are not the same ones everywhere)
        int c = gr.n_pre + c0;
        row_tile<HD> t;
        load_query_tile<HD>(a.q, a.anc_mask, r0, rt, R, G, a.hq, j, lane >> 5, lane & 31, t.qf, t.anc);
        t.lo = 0;
        t.hi = s.L;
        begin_tile<HD>(t);
        ring_keys<HD, true, true>(a, s, bt, j, k0, k_end, part_keys, 0, s.L, t, rt >= nrt, lds, [&]() __attribute__((always_inline)) {
            if (!direct) {
                put_partial<HD>(a, t, r0, rt, R, G, j, c, lane);
                begin_tile<HD>(t);
                c++;
            }
        });
        if (direct) put_result<HD>(a, t, r0, rt, R, G, j, lane);
    }
}

// Workgroups for own keys, which memory bounds, and behind them those for prefixes, which the matrix unit bounds: the ones' loads and the others'
// products overlap.  (Prefixes in front: the drafts 184 us instead of 163, the trees 213 instead of 209.)
template <int HD>
__global__ __launch_bounds__(256, 2) void shared_rows(shr_args a) {
    __shared__ __attribute__((aligned(1024))) win_lds<HD> lds;
    if ((int)blockIdx.x >= a.own_units) prefix_rows<HD>(a, lds);
    else own_rows<HD>(a, lds);
}

// Joins the partial results of a row's query heads in their order: a wavefront takes 512 / HD heads of a row, a lane eight elements of one, four partial
// results at a time (a prefix has three runs as a rule), all of which are asked for before the first is used.  EARLY: with few rows there may be many,
// sixteen of which are asked for before it is known how many there are, and whether there is the row: what a launch of a few rows takes is its chain
// of round trips to memory.
template <int HD, bool EARLY>
__global__ __launch_bounds__(256) void shared_merge(shr_args a) {
    constexpr int LANES = HD / 8, HEADS = 64 / LANES, AHEAD = EARLY ? 16 : 4;
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
            // (in bounds whether the row and its partial results exist or not)
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                x0[p] = ml[min(p, a.max_parts - 1) * a.part_rows];
                v0[p] = *reinterpret_cast<const f16x8*>(po + min(p, a.max_parts - 1) * a.part_rows * HD);
            }
            hs_loads_issued();
        }
        if (row >= a.row_off[a.batch]) return;
        const int n = a.parts[a.row2seq[row]];
        if (n < 0) continue;
        float top = -INFINITY, den = 0.f, acc[8];
#pragma unroll
        for (int i = 0; i < 8; i++) acc[i] = 0.f;
        for (int p0 = 0; p0 < n; p0 += AHEAD) {
            float2 x[AHEAD];
            f16x8 v[AHEAD];
#pragma unroll
            for (int p = 0; p < AHEAD; p++) {
                if (EARLY && p0 == 0) {
                    x[p] = x0[p];
                    v[p] = v0[p];
                } else if (p0 + p < n) {
                    x[p] = ml[(p0 + p) * a.part_rows];
                    v[p] = *reinterpret_cast<const f16x8*>(po + (p0 + p) * a.part_rows * HD);
                }
            }
            float m = top;
#pragma unroll
            for (int p = 0; p < AHEAD; p++)
                if (p0 + p < n) m = fmaxf(m, x[p].x);
            const float safe = m == -INFINITY ? 0.f : m;
            if (p0 > 0) {
                const float alpha = fast_exp2(top - safe);
                den *= alpha;
#pragma unroll
                for (int i = 0; i < 8; i++) acc[i] *= alpha;
            }
            top = m;
#pragma unroll
            for (int p = 0; p < AHEAD; p++)
                if (p0 + p < n) {
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
//
// Own keys are one walk per (sequence, KV head) where the limits allow as many of these as compute units and at most SHARED_WHOLE_KEYS keys behind the
// longest prefix, or so few keys that the walk is as short as a second partial result's way; else they are cut into partitions, a workgroup each as
// far as there are no more than sixteen for every compute unit.  7 sequences of up to 1900 tokens, 2 KV heads: a walk 52 us, partitions 16.  More
// sequences with 50 own tokens and more behind 1500 to 2048, 28 and 4 heads; both launches with whole walks and with partitions of 2048 keys, us:
//
//   own tokens to                      1500       2500       3500       5000       7000      10000      14000
//   128 single tokens               54   67    83   96   108  114   147  141   198  173   273  223   376  305
//   128 with drafts                 73   89    93  112   119  135   164  169   223  217   314  297   431  380
//   64 trees, 40 and 8 heads       107  117   131  136   149  162   186  192   243  247   332  319   451  419
//   10 of 128 places still taken    44   44    65   59    87   63   119   65   162   69   227   73   313   82
//
// (The limits do not tell how many places are taken.  At the end of a rollout a few long sequences walk their keys on a few compute units: up to 6000
// keys that is up to twice as long as it could be, beyond it partitions are about as fast with all places taken.)
//
// A prefix is cut into as many runs as two workgroups for every compute unit take, three at least, so that the last ones to start are short (all figures
// of this paragraph by one build, in which the trees took 209 and the drafts 163, since then 205 and 160): 64 trees
// of 17 nodes behind 8000 tokens, 8 KV heads, with 1, 2, 3, 4 and 6 runs 232, 244, 209, 224 and 232 us, the drafts 232, 176, 163, 164 and 164, single tokens
// 144, 121, 125, 127 and 129 (more runs keep the long walks of own keys waiting), 7 sequences behind 700 tokens 24, 19, 17, 16 and 16; 16 trees behind 4096
// tokens with as many runs as fit at once, five, 52, with six 59.  Where the rows alone fill the chip a run has sixteen tiles at least, since a partial
// result costs what it takes to write and read: 128 trees of 8 prompts behind 512 tokens with one run 67, with three 85; the drafts behind 512 with one 51, with
// three 48, behind 2048 as many as before.  All of this is counted by the limits and the longest prefix: decoding without drafts under limits for drafts gets
// fewer runs than it has room for, and a group with a shorter prefix as many runs as the longest, of a tile at least.
//
// With short tables nothing is shared: the prefix lies in the caches, each sequence walks it with its own keys, and there are no partial results and no
// second launch.  7 sequences of 64 + 32 tokens 8.3 us, with sharing 10.7, 128 + 64: 10.1 and 11.5, 256 + 64: 13.0 and 11.5; with many sequences
// the walks overlap: 128 single tokens 256 + 64 15.3 and 17.1, the drafts 300 + 70 44 and 43, 64 trees 300 + 70 22 and 39.  (Trees whose rows fill their tiles
// would be faster alone up to 2000 tokens, 1024 + 64: 41 and 54; the drafts, within the same limits, slower, 80 and 57.)
constexpr int SHARED_WHOLE_KEYS = 6000, SHARED_SHORT_KEYS = 160, SHARED_ALONE_MANY = 400, SHARED_ALONE_FEW = 208;
constexpr int SHARED_RUNS = 3, SHARED_RUN_TILES = 4, SHARED_RUN_TILES_MANY = 16;
struct shr_plan { int part_keys, max_parts, splits; bool whole; };
shr_plan plan_keys(const hs_ctx* ctx, const hs_shared_prefix* pre) {
    const hs_limits& l = ctx->lim;
    const hs_model_desc& d = ctx->desc;
    const long long cap = (long long)l.max_blocks_per_seq * 16, longest = std::min<long long>(pre->max_prefix, cap);
    const long long span = std::max<long long>(cap - longest, 32), pairs = (long long)l.max_batch * d.n_kv_heads;
    shr_plan p;
    p.whole = span <= (pairs >= ctx->n_cu ? SHARED_WHOLE_KEYS : SHARED_SHORT_KEYS);
    const bool alone = cap <= (2 * pairs >= ctx->n_cu ? SHARED_ALONE_MANY : SHARED_ALONE_FEW);
    p.whole |= alone;
    long long part = 2048;
    while (part > ctx->att_part && pairs * ((span + part - 1) / part) < 4ll * ctx->n_cu) part /= 2;
    p.part_keys = (int)std::max<long long>(part, ctx->att_part);      // (a table's keys in partitions of att_part: max_parts)
    p.max_parts = ctx->max_parts + hs_shared_runs(ctx);
    const long long rows = (long long)(d.n_q_heads / d.n_kv_heads) * pre->max_members * (1 + l.c_max * l.k_max), tiles = longest / 32;
    const long long units = (long long)pre->n_groups * d.n_kv_heads * ((rows + 127) / 128);
    const long long want = std::max<long long>(SHARED_RUNS, 2 * ctx->n_cu / units), least = units >= ctx->n_cu ? SHARED_RUN_TILES_MANY : SHARED_RUN_TILES;
    p.splits = tiles == 0 || alone ? 0 : (int)std::max(1ll, std::min({want, (long long)hs_shared_runs(ctx), tiles / least}));
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
        a.runs = (int)std::max(1ll, std::min(own, (16ll * ctx->n_cu + pairs - 1) / pairs));
    }
    a.own_units = a.batch * a.hkv * a.runs * a.tiles;
    a.prefix_units = (a.n_groups * a.hkv * a.splits + 7) / 8 * 8 * a.prefix_tiles;
    return a;
}

}  // namespace

// (with few rows many runs; of 64 MB, and 32, at most, and as many as every prefix has)
int hs_shared_runs(const hs_ctx* ctx) {
    const long long row = (long long)ctx->desc.n_q_heads * (ctx->desc.head_dim * 2 + 8) * ctx->lim.max_rows;
    return (int)std::min(32ll, std::max<long long>(SHARED_RUNS, (64ll << 20) / row));
}

void hs_launch_shared_attention(const hs_ctx* ctx, int layer, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step,
                                const hs_shared_prefix* pre, const void* q, void* out, hipStream_t st) {
    const shr_args a = make_args(ctx, layer, cache, seq, step, pre, q, out);
    const dim3 grid((unsigned)(a.own_units + a.prefix_units));
    if (ctx->desc.head_dim == 128) hipLaunchKernelGGL((shared_rows<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((shared_rows<64>), grid, dim3(256), 0, st, a);
}

void hs_launch_shared_merge(const hs_ctx* ctx, const hs_kv_cache* cache, const hs_seq_state* seq, const hs_step* step, const hs_shared_prefix* pre,
                            void* out, hipStream_t st) {
    const shr_args a = make_args(ctx, 0, cache, seq, step, pre, nullptr, out);
    if (a.whole && a.splits == 0) return;      // (all rows have their results)
    const int per = 4 * 512 / ctx->desc.head_dim, sets = (a.hq + per - 1) / per;      // heads of a workgroup, workgroups of a row
    const dim3 grid(hs_row_grid(ctx, 256, sets), sets);
    const bool early = ctx->lim.max_rows <= HS_EARLY_ROWS;
    if (ctx->desc.head_dim == 128) {
        if (early) hipLaunchKernelGGL((shared_merge<128, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((shared_merge<128, false>), grid, dim3(256), 0, st, a);
    } else {
        if (early) hipLaunchKernelGGL((shared_merge<64, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((shared_merge<64, false>), grid, dim3(256), 0, st, a);
    }
}
