// Log probabilities of tokens, the entropy of their distributions, and the largest alternatives.  With x_t = (l_t - max l) / T and S = sum exp(x):
//
//   log p(t) = x_t - ln S        H = ln S - sum(x exp(x)) / S        the k largest l_t, the lower token first among equal ones
//
// Bound by memory: the logits are read once.  The first launch takes a vocabulary in chunks of 8192 tokens, a workgroup each, and leaves each chunk's
// maximum, sum of exp and sum of x exp, and the largest logit of every unit of 256 tokens; the second joins the chunks in their order, in 64 bits.
// A row's k largest tokens lie in units whose maximum is not below the k-th largest one (k units have a token as large): the second launch reads little
// more than k units again.
// Chunks and units belong to the vocabulary alone: a row's results have the same bits whatever else is asked.
// 1088 rows of 152064 floats with 20 alternatives: 117 us for the first launch (5.7 TB/s, of the 6.2 that reads alone reach) and 14 for the second;
// the emitted tokens of 64 sequences, without alternatives, 20 and 3.5; 7 rows of bf16 with 5: 4.6 and 8, two chains of round trips to memory.  Logits
// of 16 bits, with as many instructions per logit, reach less of that rate: both launches with 20 alternatives, 1088 rows of 152064 90 us (3.7 TB/s), of 32000 33.
// Rows that do not begin at 16 bytes are read element by element: 1088 rows of 50257 bf16 88 us and of 50256 42, in 32 bits 67 and 58.
#include <algorithm>
#include <cmath>

#include "hs_internal.h"
#include "hs_lanes.h"

namespace {

constexpr int CHUNK = 8192, UNIT = 256, CHUNK_UNITS = CHUNK / UNIT;
constexpr int UNITS_LDS = 2048;      // a row's units in LDS; of larger vocabularies (from 524288 tokens on) they are read again from memory

struct __attribute__((aligned(16))) lp_stat { float m, s, e; };      // largest logit; sums of w and w d, w = exp2(d), d = (l - m) log2(e) / T
struct lp_args {
    const void* logits;
    size_t stride;
    int rows, vocab, n, first, top, chunks, units;      // first: the number of entry 0 of this launch
    float c;                                            // log2(e) / T
    double t;
    const int32_t *row, *token, *live;
    // emitted tokens: entry (b, i) = the i-th one of sequence b
    const int32_t *row_off, *n_out, *out_tok, *path_row;
    int k_stride, batch;
    lp_stat* stats;          // [entries of the launch][chunks]
    float* most;             // [entries of the launch][units]
    float *logprob, *entropy, *top_logprob;
    int32_t* top_token;
};

// An entry's row and token.  Row -1: nothing is asked; -2: there is no such row.
struct lp_entry { int row, token; };
__device__ __forceinline__ lp_entry entry_of(const lp_args& a, int i) {
    lp_entry e = {-1, -1};
    if (a.row_off) {
        const int b = i / a.k_stride, at = i % a.k_stride;
        if (b >= a.batch || at >= a.n_out[b]) return e;
        e.row = a.row_off[b] + a.path_row[i];
        e.token = a.out_tok[i];
    } else {
        if (a.live && i >= *a.live) return e;
        e.row = a.row ? a.row[i] : i;
        e.token = a.token[i];
    }
    if ((unsigned)e.row >= (unsigned)a.rows) e.row = -2;
    return e;
}

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return bf16_to_f32(v); }
template <typename T> constexpr int run_of = 16 / sizeof(T);
// A run of 16 bytes that begins at token i; tokens beyond the vocabulary: -inf.
template <typename T>
__device__ __forceinline__ void load_run(const T* __restrict__ row, int i, int vocab, bool aligned, float (&v)[run_of<T>]) {
    constexpr int RUN = run_of<T>;
    if (aligned && i + RUN <= vocab) {
        typedef T run_t __attribute__((ext_vector_type(RUN)));
        const run_t x = __builtin_nontemporal_load(reinterpret_cast<const run_t*>(row + i));
#pragma unroll
        for (int e = 0; e < RUN; e++) v[e] = wide((T)x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < RUN; e++) v[e] = i + e < vocab ? wide(row[i + e]) : -INFINITY;
    }
}
__device__ __forceinline__ float wave_sum_f32(float v) {
    auto step = [&](unsigned other) { v += __uint_as_float(other); };
    step(lane_xor<32>(__float_as_uint(v)));
    step(lane_xor<16>(__float_as_uint(v)));
    step(lane_xor<8>(__float_as_uint(v)));
    step(lane_xor<4>(__float_as_uint(v)));
    step(lane_xor<2>(__float_as_uint(v)));
    step(lane_xor<1>(__float_as_uint(v)));
    return v;
}

// A chunk: every lane has 32 of its tokens, in runs of 16 bytes, a wavefront's side by side: one unit of 32-bit logits, two of 16-bit ones.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_stats(lp_args a) {
    constexpr int RUN = run_of<T>, RUNS = CHUNK / 256 / RUN;
    __shared__ float s_sum[2][4], s_max[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int at = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const lp_entry q = entry_of(a, a.first + at);
    if (q.row < 0) return;
    const T* row = (const T*)a.logits + (size_t)q.row * a.stride;
    const bool aligned = ((unsigned long long)row & 15ull) == 0;
    float v[RUNS][RUN], top = -INFINITY;
#pragma unroll
    for (int r = 0; r < RUNS; r++) load_run<T>(row, chunk * CHUNK + ((r * 4 + wave) * 64 + lane) * RUN, a.vocab, aligned, v[r]);
#pragma unroll
    for (int r = 0; r < RUNS; r++) {
        float m = v[r][0];
#pragma unroll
        for (int e = 1; e < RUN; e++) m = fmaxf(m, v[r][e]);
        if (a.top > 0) {
            m = wave_max_f32<RUN == 4 ? 64 : 32>(m);
            const int unit = chunk * CHUNK_UNITS + (r * 4 + wave) * (RUN / 4) + (RUN == 4 ? 0 : lane >> 5);
            if ((lane & (RUN == 4 ? 63 : 31)) == 0 && unit < a.units) a.most[(size_t)at * a.units + unit] = m;
        }
        top = fmaxf(top, m);
    }
    top = wave_max_f32(top);
    if (lane == 0) s_max[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    // (a chunk of nothing but -inf: every weight is 0, and no difference of infinities is taken)
    const float m = top == -INFINITY ? 0.f : top;
    float s = 0.f, e2 = 0.f;
#pragma unroll
    for (int r = 0; r < RUNS; r++)
#pragma unroll
        for (int e = 0; e < RUN; e++) {
            const float d = (v[r][e] - m) * a.c, w = __builtin_amdgcn_exp2f(d);
            s += w;
            e2 += w > 0.f ? w * d : 0.f;      // (0 times an infinity; a NaN is in s)
        }
    s = wave_sum_f32(s);
    e2 = wave_sum_f32(e2);
    if (lane == 0) { s_sum[0][wave] = s; s_sum[1][wave] = e2; }
    __syncthreads();
    if (tid == 0)
        a.stats[(size_t)at * a.chunks + chunk] = {top, (s_sum[0][0] + s_sum[0][1]) + (s_sum[0][2] + s_sum[0][3]),
                                                  (s_sum[1][0] + s_sum[1][1]) + (s_sum[1][2] + s_sum[1][3])};
}

// Keys in the order of what is looked for: larger values first, then lower numbers; no two are equal, and 0 is none.
typedef unsigned long long u64;
__device__ __forceinline__ unsigned ordered(float v) {
    const unsigned u = __float_as_uint(v + 0.f);      // (-0 is 0)
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 key_of(float v, int number) { return ((u64)ordered(v) << 32) | (0xFFFFFFFFu - (unsigned)number); }
__device__ __forceinline__ float value_of(unsigned u) { return __uint_as_float((u & 0x80000000u) ? u & 0x7FFFFFFFu : ~u); }
__device__ __forceinline__ int key_number(u64 k) { return (int)(0xFFFFFFFFu - (unsigned)k); }
template <int O>
__device__ __forceinline__ void max_step(u64& k) {
    const u64 other = ((u64)lane_xor<O>((unsigned)(k >> 32)) << 32) | lane_xor<O>((unsigned)k);
    k = other > k ? other : k;
}
__device__ __forceinline__ u64 wave_max_key(u64 k) {
    max_step<32>(k);
    max_step<16>(k);
    max_step<8>(k);
    max_step<4>(k);
    max_step<2>(k);
    max_step<1>(k);
    return k;
}

// What of a row's tokens is in the running is narrowed in steps that cost the same whatever k is.  128 pairs of threads look at a share each; the k-th largest
// of their maxima is a lower bound of the k-th largest of all, and little more than k values are above it.  So: the units whose maximum
// is not below such a bound, of these units' tokens those that are not (or, if still too many, not below the bound of their own), and
// for each of these the number that are in front of it.  Where more are left than there is room for, because hundreds of logits are equal, they are
// taken one by one.  (One by one for all rows, 20 of 1088 rows' 152064 logits took both launches 208 us, in these steps 141; 5 of 7 rows 18.3 and 15.2.)
constexpr int LEFT = 256;      // units or tokens in the running
struct pick_lds {
    unsigned most[256], pair[128];      // a thread's maximum in its order; a pair's, the last bits the pair's number
    unsigned bound;
    int n_units, n_tokens;
    int unit[LEFT];
    u64 token[LEFT], out[HS_LOGPROBS_TOP], red[2][4];
};
// A lower bound of the k-th largest of the pairs' maxima (ordered, 0: fewer than k have one), which 7 of the 32 bits more would make exact.  (By pairs of
// threads and two of the four wavefronts: the bound of 256 maxima is a little higher and takes four times as many instructions.)
// meanwhile(): for the last wavefront, which has nothing else to do.
template <typename Meanwhile>
__device__ __forceinline__ unsigned lower_bound(float m, int k, pick_lds& l, Meanwhile meanwhile) {
    const int tid = threadIdx.x;
    const unsigned none = ordered(-INFINITY);
    l.most[tid] = ordered(m);
    if (tid == 0) l.bound = 0;
    __syncthreads();
    const unsigned top = tid < 128 ? max(l.most[tid], l.most[tid + 128]) : 0u, mine = (top & ~127u) | (unsigned)tid;
    if (tid < 128) l.pair[tid] = mine;
    __syncthreads();
    if (tid < 128) {
        int in_front = 0;
        const uint4* all = reinterpret_cast<const uint4*>(l.pair);
#pragma unroll 16
        for (int i = 0; i < 32; i++) {
            const uint4 x = all[i];
            in_front += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
        }
        if (in_front == k - 1 && top > none) l.bound = max(top & ~127u, none + 1);
    } else if (tid >= 192) {
        meanwhile();
    }
    __syncthreads();
    return l.bound;
}
// (what a bound lets through; without one: whatever is not excluded)
__device__ __forceinline__ bool in_running(float v, unsigned bound) { return ordered(v) >= (bound ? bound : ordered(-INFINITY) + 1); }

// The k first keys of those that get(i), i < n, gives the workgroup's threads, one after the other: a thread holds its largest one, and the thread whose
// key is the largest of all looks for its next.
template <typename Get>
__device__ void one_by_one(int k, int n, Get get, pick_lds& l) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 best = 0;
    for (int i = 0; i < n; i++) {
        const u64 x = get(i);
        best = x > best ? x : best;
    }
    for (int j = 0; j < k; j++) {
        const u64 w = wave_max_key(best);
        if (lane == 0) l.red[j & 1][wave] = w;
        __syncthreads();
        u64 top = l.red[j & 1][0];
#pragma unroll
        for (int x = 1; x < 4; x++) top = l.red[j & 1][x] > top ? l.red[j & 1][x] : top;
        if (tid == 0) l.out[j] = top;
        if (best == top && top != 0) {
            best = 0;
            for (int i = 0; i < n; i++) {
                const u64 x = get(i);
                if (x < top && x > best) best = x;
            }
        }
    }
    __syncthreads();
}

// The k first tokens of a row into l.out, in order.  unit(u): the largest logit of unit u; meanwhile(): see lower_bound.
template <typename T, typename Unit, typename Meanwhile>
__device__ __forceinline__ void pick_tokens(const T* __restrict__ row, int vocab, int units, int k, Unit unit, pick_lds& l, Meanwhile meanwhile) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid == 0) l.n_units = l.n_tokens = 0;
    float m = -INFINITY;
    for (int u = tid; u < units; u += 256) m = fmaxf(m, unit(u));
    unsigned bound = lower_bound(m, k, l, meanwhile);
    for (int u = tid; u < units; u += 256)
        if (in_running(unit(u), bound)) {
            const int at = atomicAdd(&l.n_units, 1);
            if (at < LEFT) l.unit[at] = u;
        }
    __syncthreads();
    const int n_units = l.n_units;
    const bool aligned = ((unsigned long long)row & 15ull) == 0;
    auto token = [&](int q) { return l.unit[q] * UNIT + tid; };
    auto logit = [&](int q) { return token(q) < vocab ? wide(row[token(q)]) : -INFINITY; };
    bool fits = n_units <= LEFT;
    for (int turn = 0; fits; turn++) {
        if (turn == 1) {      // too many: the bound of these tokens themselves
            float most = -INFINITY;
#pragma unroll 4
            for (int q = 0; q < n_units; q++) most = fmaxf(most, logit(q));
            if (tid == 0) l.n_tokens = 0;
            bound = max(bound, lower_bound(most, k, l, [] {}));
        }
        if (turn == 0 && bound == 0 && n_units > 1) continue;      // (no bound: that of the tokens at once)
        // Thirty-two units on their way, a wavefront has whole ones in runs of 16 bytes: they are no longer in the caches, and a trip to memory takes longer
        // than the rest.  (A token per thread and sixteen units on their way: 1088 rows of 152064 floats, 20 alternatives, 141 us, so 136; 128 rows 39 and 34;
        // 7 rows 16 and 14; 1088 rows of 32000 bf16 logits 41 and 33.)
        constexpr int RUN = run_of<T>, PER = 64 * RUN / UNIT, LOADS = 8 / PER;
        for (int q0 = 0; q0 < n_units; q0 += 32) {
            float v[LOADS][RUN];
            const bool second = q0 + 16 < n_units;      // (with few alternatives there are no more than sixteen)
            auto first = [&](int r) {
                const int q = q0 + (r * 4 + (tid >> 6)) * PER + lane * PER / 64;
                return q < n_units ? l.unit[q] * UNIT + lane * RUN % UNIT : vocab;
            };
            auto load = [&](int r0) {
#pragma unroll
                for (int r = r0; r < r0 + LOADS / 2; r++) load_run<T>(row, first(r), vocab, aligned, v[r]);
            };
            auto take = [&](int r0) {
#pragma unroll
                for (int r = r0; r < r0 + LOADS / 2; r++)
#pragma unroll
                    for (int e = 0; e < RUN; e++)
                        if (in_running(v[r][e], bound)) {
                            const int at = atomicAdd(&l.n_tokens, 1);
                            if (at < LEFT) l.token[at] = key_of(v[r][e], first(r) + e);
                        }
            };
            load(0);
            if (second) load(LOADS / 2);
            take(0);
            if (second) take(LOADS / 2);
        }
        __syncthreads();
        if (l.n_tokens <= LEFT) break;
        __syncthreads();
        fits = turn == 0;
    }
    if (fits) {
        const int n = l.n_tokens;
        if (tid < n) {
            const u64 mine = l.token[tid];
            int in_front = 0;
#pragma unroll 4
            for (int i = 0; i < n; i++) in_front += l.token[i] > mine;
            if (in_front < k) l.out[in_front] = mine;
        }
        // fewer than k that are not excluded: the first excluded tokens follow, which are among the first n + k
        if (n < k && tid < 64) {
            const bool gone = lane < vocab && wide(row[lane]) == -INFINITY;
            const int at = n + __popcll(__ballot(gone) & ((1ull << lane) - 1));
            if (gone && at < k) l.out[at] = key_of(-INFINITY, lane);
        }
        __syncthreads();
        return;
    }
    one_by_one(min(k, units), (units + 255) / 256, [&](int j) { const int u = tid + 256 * j; return u < units ? key_of(unit(u), u) : 0ull; }, l);
    if (tid < min(k, units)) l.unit[tid] = key_number(l.out[tid]);
    __syncthreads();
    one_by_one(k, min(k, units), [&](int q) { return token(q) < vocab ? key_of(logit(q), token(q)) : 0ull; }, l);
}
static_assert(2 * HS_LOGPROBS_TOP <= 64, "the first excluded tokens, by a wavefront");

// An entry: the chunks joined, and what is asked of it.  Eight workgroups per compute unit, so that 2048 rows are one round of them (20 of 32000 bf16 logits
// 57 us, with five per compute unit 70; up to 1088 rows the same).
template <typename T>
__global__ __launch_bounds__(256, 8) void logprobs_join(lp_args a) {
    __shared__ float s_most[UNITS_LDS];
    __shared__ __attribute__((aligned(16))) pick_lds l;
    __shared__ double row_ln_s;
    __shared__ float row_m;
    __shared__ bool row_bad;      // (a NaN or +inf)
    const int tid = threadIdx.x, lane = tid & 63;
    const lp_entry q = entry_of(a, a.first + blockIdx.x);
    if (q.row == -1) return;
    const size_t i = (size_t)a.first + blockIdx.x;
    const T* row = (const T*)a.logits + (size_t)max(q.row, 0) * a.stride;
    const lp_stat* st = a.stats + (size_t)blockIdx.x * a.chunks;
    const float nan = __uint_as_float(0x7FC00000u);
    if (q.row < 0) {
        if (tid == 0) {
            a.logprob[i] = nan;
            if (a.entropy) a.entropy[i] = nan;
        }
        if (tid < a.top) {
            a.top_token[i * a.top + tid] = -1;
            a.top_logprob[i * a.top + tid] = nan;
        }
        return;
    }
    // The chunks, by one wavefront, which has asked for the first ones (and for the token's logit) before it is its turn.  (What is picked from a row with
    // a NaN or +inf is not used.)
    const lp_stat x0 = lane < a.chunks ? st[lane] : lp_stat{-INFINITY, 0.f, 0.f};
    const float own = (unsigned)q.token < (unsigned)a.vocab ? wide(row[q.token]) : -INFINITY;
    auto join_chunks = [&]() {
        float m = x0.m;
        for (int c = lane + 64; c < a.chunks; c += 64) m = fmaxf(m, st[c].m);
        m = wave_max_f32(m);
        double s = 0., e = 0.;
        auto add = [&](const lp_stat& x) {
            const float d = x.m == -INFINITY ? 0.f : (x.m - m) * a.c, w = __builtin_amdgcn_exp2f(d);
            s += (double)w * x.s;
            e += (double)w * x.e + (w > 0.f ? (double)d * w * x.s : 0.);
        };
        add(x0);
        for (int c = lane + 64; c < a.chunks; c += 64) add(st[c]);
        s = wave_sum_f64(s);
        e = wave_sum_f64(e);
        const bool bad = !(s < INFINITY) || m == INFINITY, none = m == -INFINITY;
        const double ln_s = bad || none ? 0. : log(s);
        if (lane == 0) {
            row_m = m;
            row_ln_s = ln_s;
            row_bad = bad;
            a.logprob[i] = bad ? nan : own == -INFINITY ? -INFINITY : (float)(((double)own - m) / a.t - ln_s);
            if (a.entropy) a.entropy[i] = bad ? nan : none ? 0.f : (float)(ln_s - e / s * 0.6931471805599453);
        }
    };
    if (a.top == 0) {
        if (tid < 64) join_chunks();
        return;
    }
    const float* most = a.most + (size_t)blockIdx.x * a.units;
    if (a.units <= UNITS_LDS) {
        for (int u = tid; u < a.units; u += 256) s_most[u] = most[u];
        __syncthreads();
        pick_tokens(row, a.vocab, a.units, a.top, [&](int u) { return s_most[u]; }, l, join_chunks);
    } else {
        pick_tokens(row, a.vocab, a.units, a.top, [&](int u) { return most[u]; }, l, join_chunks);
    }
    if (tid < a.top) {      // (behind a barrier of pick_tokens)
        const u64 key = l.out[tid];
        const float v = value_of((unsigned)(key >> 32));
        const bool bad = row_bad;
        a.top_token[i * a.top + tid] = bad ? -1 : key_number(key);
        a.top_logprob[i * a.top + tid] = bad ? nan : v == -INFINITY ? -INFINITY : (float)(((double)v - row_m) / a.t - row_ln_s);
    }
}

}  // namespace

size_t hs_logprobs_scratch(int vocab) {
    // what a call needs per entry; room for 16 MB of them, and for one at least
    const size_t chunks = ((size_t)vocab + CHUNK - 1) / CHUNK, units = ((size_t)vocab + UNIT - 1) / UNIT;
    return std::max<size_t>(16u << 20, chunks * sizeof(lp_stat) + units * 4);
}

void hs_launch_logprobs(const hs_ctx* ctx, const hs_logprobs_args* args, const hs_seq_state* seq, const hs_step* step, const void* logits,
                        long long stride, int type, int rows, hipStream_t st) {
    lp_args a = {};
    a.logits = logits;
    a.stride = (size_t)stride;
    a.rows = rows;
    a.vocab = ctx->desc.vocab;
    a.top = args->top;
    a.chunks = (a.vocab + CHUNK - 1) / CHUNK;
    a.units = (a.vocab + UNIT - 1) / UNIT;
    a.t = (double)args->temperature;
    a.c = (float)(1.4426950408889634 / a.t);
    a.row = args->row;
    a.token = args->token;
    a.live = args->live;
    a.n = args->n;
    if (args->emitted) {
        a.row_off = step->row_off;
        a.n_out = step->n_out;
        a.out_tok = step->out_tok;
        a.path_row = step->path_row;
        a.k_stride = ctx->lim.k_max + 1;
        a.batch = seq->batch;
        a.n = a.batch * a.k_stride;
    }
    a.logprob = args->logprob;
    a.entropy = args->entropy;
    a.top_token = args->top_token;
    a.top_logprob = args->top_logprob;
    const size_t per = a.chunks * sizeof(lp_stat) + (a.top > 0 ? (size_t)a.units * 4 : 0);
    const int most = (int)std::min<size_t>(hs_logprobs_scratch(a.vocab) / per, (1u << 23) / a.chunks);      // (a grid has fewer than 2^24 workgroups of 256)
    char* scratch = ctx->ws + ctx->lay.logprobs;
    for (long long first = 0; first < a.n; first += most) {
        a.first = (int)first;
        const int n = std::min(most, a.n - a.first);
        a.stats = (lp_stat*)scratch;
        a.most = (float*)(scratch + (size_t)n * a.chunks * sizeof(lp_stat));
        if (type == HS_F32) {
            hipLaunchKernelGGL((logprobs_stats<float>), dim3(n * a.chunks), dim3(256), 0, st, a);
            hipLaunchKernelGGL((logprobs_join<float>), dim3(n), dim3(256), 0, st, a);
        } else {
            hipLaunchKernelGGL((logprobs_stats<bf16_t>), dim3(n * a.chunks), dim3(256), 0, st, a);
            hipLaunchKernelGGL((logprobs_join<bf16_t>), dim3(n), dim3(256), 0, st, a);
        }
    }
}
