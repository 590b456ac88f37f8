// Probabilities: the softmax of a step's logits, and the verification of drafted tokens against the target's (and the draft's)
// probabilities with random numbers that the caller gives.
#include <algorithm>
#include <cmath>

#include "hs_internal.h"
#include "hs_lanes.h"

namespace {

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void narrow(float v, float& to) { to = v; }
__device__ __forceinline__ void narrow(float v, bf16_t& to) { to = __builtin_isnan(v) ? (bf16_t)0x7FC0 : f32_to_bf16(v); }

// Rows are read and written in runs of 16 bytes of the logits, a wavefront's side by side: with eight values of 32 bits per lane, in two halves,
// every access of the wavefront's touched half of twice as many sectors (1088 rows of 152064 tokens 336 -> 316 us).
// (Stores are non-temporal: what they would take of the caches is better used by logits that are read again, 390 -> 357 us for 1088 rows of
// 152064 tokens when a workgroup read all of its row twice.)
template <typename T> constexpr int run_of = 16 / sizeof(T);
// PER tokens, in runs that begin at from, from + step, ...  all: 16-byte accesses are possible, and all of the tokens are in the row (the same for
// the wavefront: its loads are issued one after the other, without branches between them).
template <int PER, typename T>
__device__ __forceinline__ void load_runs(const T* __restrict__ row, int from, int step, int n, bool all, float rest, float (&v)[PER]) {
    constexpr int RUN = run_of<T>;
    if (all) {
        typedef T run_t __attribute__((ext_vector_type(RUN)));
#pragma unroll
        for (int u = 0; u < PER / RUN; u++) {
            const run_t x = *reinterpret_cast<const run_t*>(row + from + u * step);
#pragma unroll
            for (int e = 0; e < RUN; e++) v[u * RUN + e] = wide((T)x[e]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; j++) {
            const int i = from + j / RUN * step + j % RUN;
            v[j] = i < n ? wide(row[i]) : rest;
        }
    }
}
template <int RUN, typename T>
__device__ __forceinline__ void store_run(T* __restrict__ row, int i, int n, bool whole, const float* v) {
    if (whole && i + RUN <= n) {
        constexpr int N = RUN < run_of<T> ? RUN : run_of<T>;      // (bf16 made of floats: 8 bytes; floats made of bf16: twice 16)
        typedef T run_t __attribute__((ext_vector_type(N)));
#pragma unroll
        for (int k = 0; k < RUN; k += N) {
            run_t x;
#pragma unroll
            for (int e = 0; e < N; e++) { T y; narrow(v[k + e], y); x[e] = y; }
            __builtin_nontemporal_store(x, reinterpret_cast<run_t*>(row + i + k));
        }
    } else {
#pragma unroll
        for (int e = 0; e < RUN; e++)
            if (i + e < n) narrow(v[e], row[i + e]);
    }
}
template <typename T>
__device__ __forceinline__ bool whole_runs(const void* p, size_t stride) {
    return (((unsigned long long)p | stride * sizeof(T)) & 15ull) == 0;
}

// ---- p[t] = exp((l[t] - max l) / T) / sum.  Bound by memory: the logits once and the probabilities once, and of the second reading of the
// logits, when maximum and sum are known, what the caches don't have.  (1088 rows of 152064 tokens: 315 us, 4.2 TB/s of what has to move once, where
// a copy reaches 4.9; seven rows of bf16: 12 us, two launches.)

// Maximum and sum are those of units of 1024 tokens, a wavefront each, joined in their order: a row's probabilities have the same bits whatever
// other rows there are and however the call is launched.
constexpr int UNIT = 1024, UNIT_PER = UNIT / 64;
struct probs_args {
    const void* logits;
    void* out;
    size_t logits_stride, out_stride;
    const int32_t* live;      // rows that there are, or null: all
    int rows, vocab, units, first;      // first: the number of row 0 in what live counts
    float c_hi, c_lo;         // log2(e) / T
    float2* stats;            // [rows][units]: a unit's largest logit and the sum of its weights relative to that
};

// exp((l - m) / T): the exponent is a product of two parts, so that it is as exact as its result (a product rounded once is off by
// 2^-24 of an exponent of a hundred)
__device__ __forceinline__ float weight(float l, float m, float c_hi, float c_lo) {
    const float d = l - m, hi = d * c_hi, lo = __builtin_fmaf(d, c_hi, -hi) + d * c_lo;
    const float e = __builtin_amdgcn_exp2f(hi);
    // (an excluded logit at an infinite temperature; an exponent whose second part has lost its meaning)
    return d == -INFINITY || hi < -160.f ? 0.f : __builtin_fmaf(e * 0.6931471805599453f, lo, e);
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
// A wavefront's unit of a row (tokens beyond the vocabulary: -inf), run k of lane l at (64 k + l) RUN, and what goes into the sums.
template <typename T>
__device__ __forceinline__ void load_unit(const T* l, int unit, int lane, const probs_args& p, bool whole, float (&v)[UNIT_PER]) {
    load_runs(l, unit * UNIT + lane * run_of<T>, 64 * run_of<T>, p.vocab, whole && (unit + 1) * UNIT <= p.vocab, -INFINITY, v);
}
__device__ __forceinline__ float2 unit_stat(const float (&v)[UNIT_PER], const probs_args& p) {
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int e = 0; e < UNIT_PER; e++) m = fmaxf(m, v[e]);
    m = wave_max_f32(m);
#pragma unroll
    for (int e = 0; e < UNIT_PER; e++) s += v[e] == -INFINITY ? 0.f : weight(v[e], m, p.c_hi, p.c_lo);
    return make_float2(m, wave_sum_f32(s));
}
// The row's largest logit, and 1 / the sum of its weights, by a wavefront from the units'.
__device__ __forceinline__ float2 join_units(const float2* stats, const probs_args& p, int lane) {
    float m = -INFINITY, s = 0.f;
    for (int i = lane; i < p.units; i += 64) m = fmaxf(m, stats[i].x);
    m = wave_max_f32(m);
    for (int i = lane; i < p.units; i += 64) {
        const float2 x = stats[i];
        s += x.x == -INFINITY ? x.y : x.y * weight(x.x, m, p.c_hi, p.c_lo);
    }
    s = wave_sum_f32(s);
    return make_float2(m, s == 0.f ? 0.f : 1.f / s);
}
template <typename TI, typename T>
__device__ __forceinline__ void store_unit(T* o, int unit, int lane, const probs_args& p, bool whole, float (&v)[UNIT_PER], float2 top) {
    constexpr int RUN = run_of<TI>;
#pragma unroll
    for (int k = 0; k < UNIT_PER / RUN; k++) {
#pragma unroll
        for (int e = k * RUN; e < (k + 1) * RUN; e++) v[e] = (v[e] == -INFINITY ? 0.f : weight(v[e], top.x, p.c_hi, p.c_lo)) * top.y;
        store_run<RUN>(o, unit * UNIT + (64 * k + lane) * RUN, p.vocab, whole, v + k * RUN);
    }
}

// Many rows: a workgroup each, which takes its second pass from the row's end to its start, the last part first that the caches still have.
// One workgroup per compute unit, so that the rows at hand (256 of 608 KB) stay in the 256 MB of the last cache.  (With 57344 tokens in registers
// and 32768 in LDS between the passes 1088 rows took 381 us instead of 357: the caches are good enough, and the wavefronts are better off.)
constexpr int ROW_UNITS = 4096;      // a row's units in LDS
template <typename TI, typename TO>
__global__ __launch_bounds__(1024) void probs_rows(probs_args p) {
    __shared__ float2 stats[ROW_UNITS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int M = p.live ? min(*p.live, p.rows) : p.rows;
    const bool in_whole = whole_runs<TI>(p.logits, p.logits_stride), out_whole = whole_runs<TO>(p.out, p.out_stride);
    for (int row = blockIdx.x; row < M; row += gridDim.x) {
        const TI* l = (const TI*)p.logits + row * p.logits_stride;
        TO* o = (TO*)p.out + row * p.out_stride;
        __syncthreads();      // (the row before has been read)
        for (int k = wave; k < p.units; k += 32) {
            float v[2][UNIT_PER];
            load_unit(l, k, lane, p, in_whole, v[0]);
            if (k + 16 < p.units) load_unit(l, k + 16, lane, p, in_whole, v[1]);
            float2 x = unit_stat(v[0], p);
            if (lane == 0) stats[k] = x;
            if (k + 16 < p.units) {
                x = unit_stat(v[1], p);
                if (lane == 0) stats[k + 16] = x;
            }
        }
        __syncthreads();
        const float2 top = join_units(stats, p, lane);
        for (int k = (p.units - 1) / 16 * 16 + wave; k >= 0; k -= 16) {
            if (k >= p.units) continue;
            float v[UNIT_PER];
            load_unit(l, k, lane, p, in_whole, v);
            store_unit<TI>(o, k, lane, p, out_whole, v, top);
        }
    }
}

// Few rows: a workgroup per four units; one launch for the units' maxima and sums, one that joins them and writes.
template <typename TI>
__global__ __launch_bounds__(256) void probs_stats(probs_args p) {
    const int groups = (p.units + 3) / 4, row = blockIdx.x / groups, lane = threadIdx.x & 63;
    const int unit = blockIdx.x % groups * 4 + (threadIdx.x >> 6);
    if (unit >= p.units || (p.live && p.first + row >= *p.live)) return;
    float v[UNIT_PER];
    load_unit((const TI*)p.logits + row * p.logits_stride, unit, lane, p, whole_runs<TI>(p.logits, p.logits_stride), v);
    const float2 x = unit_stat(v, p);
    if (lane == 0) p.stats[(size_t)row * p.units + unit] = x;
}
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void probs_write(probs_args p) {
    const int groups = (p.units + 3) / 4, row = blockIdx.x / groups, lane = threadIdx.x & 63;
    const int unit = blockIdx.x % groups * 4 + (threadIdx.x >> 6);
    if (unit >= p.units || (p.live && p.first + row >= *p.live)) return;
    float v[UNIT_PER];
    load_unit((const TI*)p.logits + row * p.logits_stride, unit, lane, p, whole_runs<TI>(p.logits, p.logits_stride), v);
    const float2 top = join_units(p.stats + (size_t)row * p.units, p, lane);
    store_unit<TI>((TO*)p.out + row * p.out_stride, unit, lane, p, whole_runs<TO>(p.out, p.out_stride), v, top);
}

// ---- verification.  At a node with the target's probabilities p and the draft's q: w_0 = p, Z_0 = 1; the children are tried in node
// order, child number k (token t, number u) is accepted where u Z_k q(t) < w_k(t); a rejected one leaves
//   w_{k+1} = max(w_k - Z_k q, 0),  Z_{k+1} = the sum of w_{k+1}
// (without q: w_{k+1} is w_k without t, and 1 stands for q(t)).  The walk ends at the node where no child is accepted, with the first
// token at which the running sum of w exceeds u Z.  All of it in 64 bits: a 32-bit p, q or u is exact there.
//
// The walk itself needs a few probabilities per node and no sums, unless a second child of a node is tried; what takes time is the sum over
// the vocabulary at the node where it ends.  So the first launch lets every workgroup of a sequence walk for itself and then sum its
// slice of the vocabulary; the last one walks again with the sums at hand and looks for the token.  A walk that needs the sum of a rejected
// child's node on its way takes a further launch of the first kind; more of these than were launched are summed by the last one alone.  (Where
// the walk has come to is recorded, so that the last launch need not walk again as a rule: a chain of round trips to memory less.)
// Bound by memory where batches are large, by the launches and their chains of round trips where they are small: 128 histories of 152064 tokens
// 18 us for the sums (4.3 TB/s) and 6 for the pick, 64 trees twice 12 to 17 and 6; four drafts over 4096 tokens 5 and 6.
constexpr int SLICE = HS_PROBS_SLICE, PER = SLICE / 256;

struct verify_record;
struct verify_args {
    const int32_t *row_off, *tok, *parent;
    const void *p, *q;
    size_t p_stride, q_stride;
    const float *u_accept, *u_sample;
    int batch, vocab, n_slices, k_stride, rounds;
    double* sums;      // [rounds][batch][n_slices]
    verify_record* records;      // [rounds][batch]
    int32_t *accept_len, *n_out, *out_tok, *path_row;
};

// A probability as it counts: what is no positive finite number has none.
__device__ __forceinline__ double counted(float v) { return v > 0.f && v < INFINITY ? (double)v : 0.0; }

// What the walk may ask of a sequence's nodes, a node per lane.
struct verify_nodes {
    int par, tok;
    double w, q, u;      // at the parent: the target's and the draft's probability of the token; the node's number
};
template <typename T>
__device__ __forceinline__ verify_nodes load_nodes(const verify_args& a, int r0, int nn, int lane) {
    verify_nodes n = {-1, -1, 0.0, 0.0, 0.0};
    if (lane > 0 && lane < nn) {
        n.par = a.parent[r0 + lane];
        n.tok = a.tok[r0 + lane];
        n.u = (double)a.u_accept[r0 + lane];
        if (n.par < 0 || n.par >= nn) n.par = -1;
        else if (n.tok >= 0 && n.tok < a.vocab) {
            n.w = counted(wide(((const T*)a.p)[(size_t)(r0 + n.par) * a.p_stride + n.tok]));
            n.q = a.q ? counted(wide(((const T*)a.q)[(size_t)(r0 + n.par) * a.q_stride + n.tok])) : 1.0;
        }
    }
    return n;
}

// (the lane is the same for the whole wavefront: no trip through the LDS unit, of which a walk would make a dozen per node)
__device__ __forceinline__ double from_lane(double v, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// Where a walk has come to: node cur after a accepted tokens and r rejected ones there.  Lane k < r: the k-th one (rej) and the sum that it
// was tried with (z); lane k: the k-th accepted node (path, from 1 on) and token (out).  ask: the number of the sum that the walk needs
// next, or of the one that its sample is drawn from.
struct verify_walk {
    int cur, a, r, rej, path, out, ask;
    double z;
    bool done;      // that sum is known, and the walk has ended
    bool last;      // it is the sum that the sample is drawn from
};
// total(i): the i-th sum that the walk asked for, of which `known` are there.
template <typename Total>
__device__ __forceinline__ verify_walk walk_drafts(const verify_nodes& n, int nn, int k_stride, bool point, int known, Total total,
                                                   int lane) {
    verify_walk s = {0, 0, 0, -1, 0, 0, 0, 1.0, false, false};
    double w = n.w;
    unsigned long long tried = 0;
    for (;;) {
        const unsigned long long kids = __ballot(n.par == s.cur) & ~tried;
        if (!kids || s.a + 1 >= k_stride) break;
        const int c = __ffsll(kids) - 1;
        double z = 1.0;
        if (s.r > 0) {
            if (s.ask >= known) return s;
            z = total(s.ask++);
        }
        const int t = __builtin_amdgcn_readlane(n.tok, c);
        if (from_lane(n.u, c) * z * from_lane(n.q, c) < from_lane(w, c)) {
            if (lane == s.a) s.out = t;
            s.cur = c;
            s.a++;
            if (lane == s.a) s.path = c;
            s.r = 0;
            tried = 0;
        } else {
            tried |= 1ull << c;
            if (n.par == s.cur) w = point ? (n.tok == t ? 0.0 : w) : fmax(w - z * n.q, 0.0);
            if (lane == s.r) { s.rej = t; s.z = z; }
            s.r++;
        }
    }
    s.last = true;
    if (s.ask >= known) return s;
    if (!(total(s.ask) > 0.0)) {      // nothing is left: the sample is the target's own
        s.r = 0;
        if (++s.ask >= known) return s;
    }
    s.done = true;
    return s;
}

struct verify_left { double z[HS_MAX_NODES]; int rej[HS_MAX_NODES]; };
__device__ __forceinline__ void publish(const verify_walk& s, verify_left& l, int tid) {      // by the first wavefront, whose walk it is
    if (tid < HS_MAX_NODES) { l.z[tid] = s.z; l.rej[tid] = s.rej; }
}
// Where the walk of a round has come to, for the kernel that picks the token: what is there says that it need not walk for itself.
enum { RECORD_MORE = 0, RECORD_LAST = 1, RECORD_BEFORE = 2 };      // the round's sum is not the last one; it is; an earlier round's was
struct alignas(16) verify_record {
    int cur, a, r, kind;
    int rej[HS_MAX_NODES], path[HS_MAX_NODES], out[HS_MAX_NODES];
    double z[HS_MAX_NODES];
};
static_assert(sizeof(verify_record) <= HS_PROBS_RECORD, "the workspace's share");

// What is left of the weights of a thread's tokens in a slice after r rejections at a node: runs of tokens, the first at `from`, `step` apart.
template <typename T>
__device__ __forceinline__ void weights_left(const verify_args& a, int row, int slice, int from, int step, int r, const verify_left& l, double (&w)[PER]) {
    constexpr int RUN = run_of<T>;
    const bool point = a.q == nullptr, draft = !point && r > 0;
    const bool pv = whole_runs<T>(a.p, a.p_stride), qv = whole_runs<T>(a.q, a.q_stride);
    const T *pr = (const T*)a.p + row * a.p_stride, *qr = (const T*)a.q + row * a.q_stride;
    float p[PER], q[PER] = {};
    const bool inside = (slice + 1) * SLICE <= a.vocab;
    load_runs(pr, from, step, a.vocab, pv && inside, 0.f, p);
    if (draft) load_runs(qr, from, step, a.vocab, qv && inside, 0.f, q);
#pragma unroll
    for (int j = 0; j < PER; j++) w[j] = counted(p[j]);
    for (int k = 0; k < r; k++) {
        const double z = l.z[k];
        const int rej = l.rej[k];
#pragma unroll
        for (int j = 0; j < PER; j++)
            w[j] = point ? (rej == from + j / RUN * step + j % RUN ? 0.0 : w[j]) : fmax(w[j] - z * counted(q[j]), 0.0);
    }
}
// Sum of one slice's weights, by the workgroup.
template <typename T>
__device__ __forceinline__ double sum_slice(const verify_args& a, int row, int slice, int r, const verify_left& l, double* red) {
    double w[PER], s = 0.0;
    weights_left<T>(a, row, slice, slice * SLICE + (int)threadIdx.x * run_of<T>, 256 * run_of<T>, r, l, w);
#pragma unroll
    for (int j = 0; j < PER; j++) s += w[j];
    return block_sum_f64(s, red);
}

// All of a row's slices, by a wavefront.
__device__ __forceinline__ double sum_slices(const double* s, int n, int lane) {
    double z = 0.0;
    for (int i = lane; i < n; i += 64) z += s[i];
    return wave_sum_f64(z);
}

template <typename T>
__global__ __launch_bounds__(256) void verify_sums(verify_args a, int round) {
    __shared__ verify_left left;
    __shared__ double red[4];
    const int b = blockIdx.y, lane = threadIdx.x & 63;
    const int r0 = a.row_off[b], nn = min(a.row_off[b + 1] - r0, HS_MAX_NODES);
    if (nn <= 0) return;
    const verify_nodes n = load_nodes<T>(a, r0, nn, lane);
    const verify_walk s = walk_drafts(n, nn, a.k_stride, a.q == nullptr, round, [&](int i) {
        return sum_slices(a.sums + ((size_t)i * a.batch + b) * a.n_slices, a.n_slices, lane);
    }, lane);
    if (blockIdx.x == 0 && threadIdx.x < 64) {
        verify_record* rec = a.records + (size_t)round * a.batch + b;
        if (lane == 0) *reinterpret_cast<int4*>(rec) = make_int4(s.cur, s.a, s.r, s.done ? RECORD_BEFORE : s.last ? RECORD_LAST : RECORD_MORE);
        rec->rej[lane] = s.rej;
        rec->path[lane] = s.path;
        rec->out[lane] = s.out;
        rec->z[lane] = s.z;
    }
    if (s.done) return;
    publish(s, left, threadIdx.x);
    __syncthreads();
    for (int slice = blockIdx.x; slice < a.n_slices; slice += gridDim.x) {
        const double z = sum_slice<T>(a, r0 + s.cur, slice, s.r, left, red);
        if (threadIdx.x == 0) a.sums[((size_t)round * a.batch + b) * a.n_slices + slice] = z;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void verify_pick(verify_args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn_lds[];
    double* own = reinterpret_cast<double*>(dyn_lds);      // [n_slices]: sums that no launch has left
    __shared__ verify_left left;
    __shared__ double red[4], totals[HS_MAX_NODES + 2], wave_tot[4];
    __shared__ int wave_first[4], wave_last[4], s_pick;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool point = a.q == nullptr;
    // Everything whose place is known, at once: the records and sums of both rounds (what has not been written is not used), the number.
    static_assert(HS_PROBS_ROUNDS == 2, "the first record or the second one");
    const int more = a.rounds > 1 ? 1 : 0;
    const verify_record *rec = a.records + b, *next = rec + (size_t)more * a.batch;
    const double *sums0 = a.sums + (size_t)b * a.n_slices, *sums1 = sums0 + (size_t)more * a.batch * a.n_slices;
    const int4 h0 = *reinterpret_cast<const int4*>(rec), h1 = *reinterpret_cast<const int4*>(next);
    const int rej0 = rec->rej[lane], path0 = rec->path[lane], out0 = rec->out[lane];
    const int rej1 = next->rej[lane], path1 = next->path[lane], out1 = next->out[lane];
    const double z0 = rec->z[lane], z1 = next->z[lane];
    const double u = (double)a.u_sample[b];
    double part0 = lane < a.n_slices ? sums0[lane] : 0.0, part1 = lane < a.n_slices ? sums1[lane] : 0.0;
    hs_loads_issued();
    const int r0 = a.row_off[b], nn = min(a.row_off[b + 1] - r0, HS_MAX_NODES);
    if (nn <= 0) {
        if (tid == 0) { a.accept_len[b] = 0; a.n_out[b] = 0; }
        return;
    }
    for (int i = lane + 64; i < a.n_slices; i += 64) { part0 += sums0[i]; part1 += sums1[i]; }
    const double total0 = wave_sum_f64(part0), total1 = wave_sum_f64(part1);
    const bool second = more && h1.w != RECORD_BEFORE;
    verify_walk s = {second ? h1.x : h0.x, second ? h1.y : h0.y, second ? h1.z : h0.z, second ? rej1 : rej0, second ? path1 : path0,
                     second ? out1 : out0, second ? 1 : 0, second ? z1 : z0, false, (second ? h1.w : h0.w) == RECORD_LAST};
    double zt = second ? total1 : total0;
    const double* sums = second ? sums1 : sums0;
    if (s.last && zt > 0.0) {
        publish(s, left, tid);
        __syncthreads();
    } else {
        if (tid == 0) { totals[0] = total0; totals[1] = total1; }
        __syncthreads();
        // more sums than there were launches for them, or nothing left: walk and sum here
        const verify_nodes n = load_nodes<T>(a, r0, nn, lane);
        for (int known = a.rounds;; known++) {
            s = walk_drafts(n, nn, a.k_stride, point, known, [&](int i) { return totals[i]; }, lane);
            __syncthreads();      // (totals, left and own have been read)
            publish(s, left, tid);
            __syncthreads();
            if (s.done) break;
            for (int i = 0; i < a.n_slices; i++) {
                const double z = sum_slice<T>(a, r0 + s.cur, i, s.r, left, red);
                if (tid == 0) own[i] = z;
            }
            __syncthreads();
            const double z = sum_slices(own, a.n_slices, lane);
            if (tid == 0) totals[known] = z;
            __syncthreads();
        }
        zt = totals[s.ask];
        sums = s.ask >= a.rounds ? own : s.ask ? sums1 : sums0;
    }
    const double target = u * zt;
    // the slice in which the running sum exceeds the target (rounding can leave it just beyond the last: that one then)
    int slice = -1, last = -1;
    double before = 0.0, upto = 0.0;
    for (int s0 = 0; s0 < a.n_slices && slice < 0; s0 += 64) {
        const double w = s0 + lane < a.n_slices ? sums[s0 + lane] : 0.0, incl = wave_prefix_f64(w, lane);
        const unsigned long long some = __ballot(w > 0.0), hit = __ballot(w > 0.0 && upto + incl > target);
        const int at = hit ? __ffsll(hit) - 1 : some ? 63 - __clzll(some) : -1;
        if (at >= 0) {
            before = upto + from_lane(incl - w, at);
            last = s0 + at;
        }
        if (hit) slice = last;
        upto += from_lane(incl, 63);
    }
    if (slice < 0) slice = last;
    if (tid == 0) s_pick = -1;
    __syncthreads();
    if (slice >= 0) {
        // PER consecutive tokens per thread: the first thread whose running sum exceeds the target holds the token
        const int lo = slice * SLICE + tid * PER;
        double w[PER], sum = 0.0;
        weights_left<T>(a, r0 + s.cur, slice, lo, run_of<T>, s.r, left, w);
#pragma unroll
        for (int j = 0; j < PER; j++) sum += w[j];
        const double incl = wave_prefix_f64(sum, lane);
        if (lane == 63) wave_tot[wave] = incl;
        __syncthreads();
        double base = before + (incl - sum);
        for (int v = 0; v < wave; v++) base += wave_tot[v];
        // (by ballots: 256 threads' atomics on one word of LDS took 4 us)
        const unsigned long long some = __ballot(sum > 0.0), hit = __ballot(sum > 0.0 && base + sum > target);
        if (lane == 0) {
            wave_first[wave] = hit ? wave * 64 + __ffsll(hit) - 1 : 256;
            wave_last[wave] = some ? wave * 64 + 63 - __clzll(some) : -1;
        }
        __syncthreads();
        const int first = min(min(wave_first[0], wave_first[1]), min(wave_first[2], wave_first[3]));
        // (rounding can leave the target just beyond the slice, or the thread's tokens: the last one with a weight then)
        if (tid == (first < 256 ? first : max(max(wave_last[0], wave_last[1]), max(wave_last[2], wave_last[3])))) {
            int pick = -1;
            bool hit = false;
#pragma unroll
            for (int j = 0; j < PER; j++) {
                base += w[j];
                if (w[j] > 0.0 && !hit) {
                    pick = lo + j;
                    hit = base > target;
                }
            }
            s_pick = pick;
        }
        __syncthreads();
    }
    if (wave == 0) {
        const int pick = s_pick >= 0 ? s_pick : a.vocab - 1;      // (no token has a probability)
        const size_t at = (size_t)b * a.k_stride + lane;
        if (lane <= s.a) {
            a.path_row[at] = s.path;      // (the root's is 0)
            a.out_tok[at] = lane < s.a ? s.out : pick;
        }
        if (lane == 0) { a.accept_len[b] = s.a; a.n_out[b] = s.a + 1; }
    }
}

// Logits that fit into the last cache are read a second time from there by a launch of their own; of more, a workgroup per row reads its row
// twice while the cache has it, in full rounds of a row per compute unit; the rest again by two launches if it fits into the cache, otherwise by a
// round of rows too, which leaves compute units without one (1088 rows of 152064 tokens: the rest in a round of rows cost 357 against 346 us;
// everything by such pairs of launches, 192 MB of logits at a time, 343 against 315).
template <typename TI, typename TO>
void launch_rows(const hs_ctx* ctx, const probs_args& all, hipStream_t st) {
    auto pairs = [&](int from, int rows) {
        for (const int per = (int)(HS_PROBS_STATS / all.units); rows > 0; from += per, rows -= per) {
            probs_args p = all;
            p.first = from;
            p.rows = std::min(rows, per);
            p.logits = (const TI*)all.logits + from * all.logits_stride;
            p.out = (TO*)all.out + from * all.out_stride;
            const dim3 grid((unsigned)p.rows * (unsigned)((p.units + 3) / 4));
            hipLaunchKernelGGL((probs_stats<TI>), grid, dim3(256), 0, st, p);
            hipLaunchKernelGGL((probs_write<TI, TO>), grid, dim3(256), 0, st, p);
        }
    };
    auto cached = [&](int rows) {
        const size_t units = (size_t)rows * all.units;
        return units * UNIT * sizeof(TI) <= HS_PROBS_CACHED && units <= HS_PROBS_STATS;
    };
    if (cached(all.rows) || all.units <= 16 || all.units > ROW_UNITS) {      // (a short row would leave most of a workgroup idle)
        pairs(0, all.rows);
    } else {
        const int rest = cached(all.rows % ctx->n_cu) ? all.rows % ctx->n_cu : 0;
        probs_args p = all;
        p.rows -= rest;
        if (p.rows > 0) hipLaunchKernelGGL((probs_rows<TI, TO>), dim3(std::min(p.rows, ctx->n_cu)), dim3(1024), 0, st, p);
        pairs(p.rows, rest);
    }
}

template <typename T>
void launch_verify(const hs_ctx* ctx, const verify_args& a, hipStream_t st) {
    // what the device holds at once, four workgroups per compute unit: each walks once, and then sums one slice after another
    const int per_seq = std::max(1, std::min(a.n_slices, 4 * ctx->n_cu / a.batch));
    for (int round = 0; round < a.rounds; round++)
        hipLaunchKernelGGL((verify_sums<T>), dim3(per_seq, a.batch), dim3(256), 0, st, a, round);
    const size_t lds = (size_t)a.n_slices * sizeof(double);
    if (lds > 48 * 1024)      // (vocabularies beyond 25 million)
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&verify_pick<T>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.batch), dim3(256), lds, st, a);
}

}  // namespace

void hs_launch_probs(const hs_ctx* ctx, const hs_probs_args* args, hipStream_t st) {
    probs_args p = {args->logits, args->out, (size_t)args->logits_stride, (size_t)args->out_stride, args->live_rows, args->rows,
                    ctx->desc.vocab, (ctx->desc.vocab + UNIT - 1) / UNIT, 0, 0.f, 0.f, reinterpret_cast<float2*>(ctx->ws + ctx->lay.probs_stats)};
    const double c = std::min(1.4426950408889634 / (double)args->temperature, 1e38);      // (finite in 32 bits, too)
    p.c_hi = (float)c;
    p.c_lo = (float)(c - (double)p.c_hi);
    const bool wide_in = args->logits_type == HS_F32, wide_out = args->out_type == HS_F32;
    if (wide_in && wide_out) launch_rows<float, float>(ctx, p, st);
    else if (wide_in) launch_rows<float, bf16_t>(ctx, p, st);
    else if (wide_out) launch_rows<bf16_t, float>(ctx, p, st);
    else launch_rows<bf16_t, bf16_t>(ctx, p, st);
}

void hs_launch_accept_probs(const hs_ctx* ctx, const hs_accept_probs_args* args, const hs_seq_state* seq, const hs_step* step,
                            hipStream_t st) {
    verify_args a = {};
    a.row_off = step->row_off; a.tok = step->tok; a.parent = step->parent;
    a.p = args->p; a.q = args->q;
    a.p_stride = (size_t)args->p_stride; a.q_stride = (size_t)args->q_stride;
    a.u_accept = args->u_accept; a.u_sample = args->u_sample;
    a.batch = seq->batch;
    a.vocab = ctx->desc.vocab;
    a.n_slices = hs_probs_slices(a.vocab);
    a.k_stride = ctx->lim.k_max + 1;
    // (a tree of two branches forks once: the sum for its second child, and the one at the end)
    a.rounds = ctx->lim.c_max > 1 ? HS_PROBS_ROUNDS : 1;
    a.sums = reinterpret_cast<double*>(ctx->ws + ctx->lay.probs_sums);
    a.records = reinterpret_cast<verify_record*>(ctx->ws + ctx->lay.probs_records);
    a.accept_len = step->accept_len; a.n_out = step->n_out; a.out_tok = step->out_tok; a.path_row = step->path_row;
    if (args->type == HS_F32) launch_verify<float>(ctx, a, st);
    else launch_verify<bf16_t>(ctx, a, st);
}
