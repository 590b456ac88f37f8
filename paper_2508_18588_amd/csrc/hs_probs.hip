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

// ---- p[t] = exp((l[t] - max l) / T) / sum: one workgroup per row, two passes over it.

struct probs_args {
    const void* logits;
    void* out;
    size_t logits_stride, out_stride;
    const int32_t* live;      // rows that there are, or null: all
    int rows, vocab;
    float c_hi, c_lo;         // log2(e) / T
};

// exp((l - m) / T): the exponent is a product of two parts, so that it is as exact as its result (a product rounded once is off by
// 2^-24 of an exponent of a hundred)
__device__ __forceinline__ float weight(float l, float m, float c_hi, float c_lo) {
    const float d = l - m, hi = d * c_hi, lo = __builtin_fmaf(d, c_hi, -hi) + d * c_lo;
    const float e = __builtin_amdgcn_exp2f(hi);
    // (an excluded logit at an infinite temperature; an exponent whose second part has lost its meaning)
    return d == -INFINITY || hi < -160.f ? 0.f : __builtin_fmaf(e * 0.6931471805599453f, lo, e);
}

template <typename TI, typename TO>
__global__ __launch_bounds__(1024) void probs_rows(probs_args p) {
    __shared__ float red_m[16], red_s[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int M = p.live ? min(*p.live, p.rows) : p.rows;
    for (int row = blockIdx.x; row < M; row += gridDim.x) {
        const TI* l = (const TI*)p.logits + row * p.logits_stride;
        TO* o = (TO*)p.out + row * p.out_stride;
        float m = -INFINITY, s = 0.f;
        for (int i = tid; i < p.vocab; i += 1024) {
            const float x = wide(l[i]);
            if (x > m) {
                s *= weight(m, x, p.c_hi, p.c_lo);
                m = x;
            }
            s += x == -INFINITY ? 0.f : weight(x, m, p.c_hi, p.c_lo);
        }
        float top = wave_max_f32(m);
        __syncthreads();      // (the row before has been read)
        if (lane == 0) red_m[wave] = top;
        __syncthreads();
        top = red_m[0];
#pragma unroll
        for (int w = 1; w < 16; w++) top = fmaxf(top, red_m[w]);
        s = m == -INFINITY ? s : s * weight(m, top, p.c_hi, p.c_lo);
#pragma unroll
        for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
        if (lane == 0) red_s[wave] = s;
        __syncthreads();
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 16; w++) sum += red_s[w];
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        for (int i = tid; i < p.vocab; i += 1024) {
            const float x = wide(l[i]);
            narrow(top == -INFINITY && x == -INFINITY ? 0.f : weight(x, top, p.c_hi, p.c_lo) * inv, o[i]);
        }
    }
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
// child's node on its way takes a further launch of the first kind; more of these than were launched are summed by the last one alone.
constexpr int SLICE = HS_PROBS_SLICE, PER = SLICE / 256;

struct verify_args {
    const int32_t *row_off, *tok, *parent;
    const void *p, *q;
    size_t p_stride, q_stride;
    const float *u_accept, *u_sample;
    int batch, vocab, n_slices, k_stride, rounds;
    double* sums;      // [rounds][batch][n_slices]
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

__device__ __forceinline__ double from_lane(double v, int lane) {
    return __hiloint2double(__shfl(__double2hiint(v), lane), __shfl(__double2loint(v), lane));
}

// Where a walk has come to: node cur after a accepted tokens and r rejected ones there.  Lane k < r: the k-th one (rej) and the sum that it
// was tried with (z); lane k: the k-th accepted node (path, from 1 on) and token (out).  ask: the number of the sum that the walk needs
// next, or of the one that its sample is drawn from.
struct verify_walk {
    int cur, a, r, rej, path, out, ask;
    double z;
    bool done;      // that sum is known, and the walk has ended
};
// total(i): the i-th sum that the walk asked for, of which `known` are there.
template <typename Total>
__device__ __forceinline__ verify_walk walk_drafts(const verify_nodes& n, int nn, int k_stride, bool point, int known, Total total,
                                                   int lane) {
    verify_walk s = {0, 0, 0, -1, 0, 0, 0, 1.0, false};
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
        const int t = __shfl(n.tok, c);
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
    if (s.ask >= known) return s;
    if (!(total(s.ask) > 0.0)) {      // nothing is left: the sample is the target's own
        s.r = 0;
        if (++s.ask >= known) return s;
    }
    s.done = true;
    return s;
}

// The 16 tokens of a slice that are thread tid's, in 16-byte pieces where rows allow them; token(j) is the j-th one's number.
template <typename T>
__device__ __forceinline__ int slice_token(int slice, int j, bool vec) {
    constexpr int N = 16 / sizeof(T);
    return slice * SLICE + (vec ? N * ((int)threadIdx.x + 256 * (j / N)) + j % N : (int)threadIdx.x + 256 * j);
}
template <typename T>
__device__ __forceinline__ void load_tokens(const T* __restrict__ row, int vocab, int slice, bool vec, float (&v)[PER]) {
    constexpr int N = 16 / sizeof(T);
    if (vec) {
#pragma unroll
        for (int j = 0; j < PER; j += N) {
            const int i = slice_token<T>(slice, j, true);
            union { uint4 u; T t[N]; } x;
            x.u = make_uint4(0u, 0u, 0u, 0u);
            if (i + N <= vocab) x.u = *reinterpret_cast<const uint4*>(row + i);
            else {
#pragma unroll
                for (int e = 0; e < N; e++)
                    if (i + e < vocab) x.t[e] = row[i + e];
            }
#pragma unroll
            for (int e = 0; e < N; e++) v[j + e] = wide(x.t[e]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; j++) {
            const int i = slice_token<T>(slice, j, false);
            v[j] = i < vocab ? wide(row[i]) : 0.f;
        }
    }
}
template <typename T>
__device__ __forceinline__ bool whole_pieces(const void* p, size_t stride) {
    return (((unsigned long long)p | stride * sizeof(T)) & 15ull) == 0;
}

// What is left of a token's weight after r rejections.
__device__ __forceinline__ double weight_left(double w, double q, int token, int r, const double* z, const int* rej, bool point) {
    for (int k = 0; k < r; k++) w = point ? (rej[k] == token ? 0.0 : w) : fmax(w - z[k] * q, 0.0);
    return w;
}

struct verify_left { double z[HS_MAX_NODES]; int rej[HS_MAX_NODES]; };
__device__ __forceinline__ void publish(const verify_walk& s, verify_left& l, int tid) {      // by the first wavefront, whose walk it is
    if (tid < HS_MAX_NODES) { l.z[tid] = s.z; l.rej[tid] = s.rej; }
}

// Sum of one slice's weights at node cur after r rejections, by the workgroup.
template <typename T>
__device__ __forceinline__ double sum_slice(const verify_args& a, int row, int slice, int r, const verify_left& l, double* red) {
    const bool point = a.q == nullptr;
    float p[PER], q[PER];
    const bool pv = whole_pieces<T>(a.p, a.p_stride), qv = point || whole_pieces<T>(a.q, a.q_stride), vec = pv && qv;
    load_tokens<T>((const T*)a.p + row * a.p_stride, a.vocab, slice, vec, p);
    if (!point && r > 0) load_tokens<T>((const T*)a.q + row * a.q_stride, a.vocab, slice, vec, q);
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < PER; j++)
        s += weight_left(counted(p[j]), !point && r > 0 ? counted(q[j]) : 0.0, slice_token<T>(slice, j, vec), r, l.z, l.rej, point);
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
    const int slice = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63;
    const int r0 = a.row_off[b], nn = min(a.row_off[b + 1] - r0, HS_MAX_NODES);
    if (nn <= 0) return;
    const verify_nodes n = load_nodes<T>(a, r0, nn, lane);
    const verify_walk s = walk_drafts(n, nn, a.k_stride, a.q == nullptr, round, [&](int i) {
        return sum_slices(a.sums + ((size_t)i * a.batch + b) * a.n_slices, a.n_slices, lane);
    }, lane);
    if (s.done) return;
    publish(s, left, threadIdx.x);
    __syncthreads();
    const double z = sum_slice<T>(a, r0 + s.cur, slice, s.r, left, red);
    if (threadIdx.x == 0) a.sums[((size_t)round * a.batch + b) * a.n_slices + slice] = z;
}

template <typename T>
__global__ __launch_bounds__(256) void verify_pick(verify_args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char dyn_lds[];
    double* own = reinterpret_cast<double*>(dyn_lds);      // [n_slices]: sums that no launch has left
    __shared__ verify_left left;
    __shared__ double red[4], totals[HS_MAX_NODES + 2], wave_tot[4];
    __shared__ int s_first, s_last, s_pick;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r0 = a.row_off[b], nn = min(a.row_off[b + 1] - r0, HS_MAX_NODES);
    if (nn <= 0) {
        if (tid == 0) { a.accept_len[b] = 0; a.n_out[b] = 0; }
        return;
    }
    const bool point = a.q == nullptr;
    const verify_nodes n = load_nodes<T>(a, r0, nn, lane);
    // (sums that the walk did not ask for have not been written: they are read, and not used)
    for (int i = wave; i < a.rounds; i += 4) {
        const double z = sum_slices(a.sums + ((size_t)i * a.batch + b) * a.n_slices, a.n_slices, lane);
        if (lane == 0) totals[i] = z;
    }
    __syncthreads();
    int known = a.rounds;
    verify_walk s;
    for (;;) {
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
        known++;
        __syncthreads();
    }
    const double* sums = s.ask < a.rounds ? a.sums + ((size_t)s.ask * a.batch + b) * a.n_slices : own;
    const double zt = totals[s.ask], target = (double)a.u_sample[b] * zt;
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
    if (tid == 0) { s_first = 256; s_last = -1; s_pick = -1; }
    __syncthreads();
    if (slice >= 0) {
        const T* pr = (const T*)a.p + (size_t)(r0 + s.cur) * a.p_stride;
        const T* qr = point ? nullptr : (const T*)a.q + (size_t)(r0 + s.cur) * a.q_stride;
        auto left_of = [&](int i) -> double {
            if (i >= a.vocab) return 0.0;
            return weight_left(counted(wide(pr[i])), !point && s.r > 0 ? counted(wide(qr[i])) : 0.0, i, s.r, left.z, left.rej, point);
        };
        // PER consecutive tokens per thread: the first thread whose running sum exceeds the target holds the token
        const int lo = slice * SLICE + tid * PER;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < PER; j++) sum += left_of(lo + j);
        const double incl = wave_prefix_f64(sum, lane);
        if (lane == 63) wave_tot[wave] = incl;
        __syncthreads();
        double base = before + (incl - sum);
        for (int q = 0; q < wave; q++) base += wave_tot[q];
        if (sum > 0.0) {
            atomicMax(&s_last, tid);
            if (base + sum > target) atomicMin(&s_first, tid);
        }
        __syncthreads();
        const int owner = s_first < 256 ? s_first : s_last;
        if (owner >= 0 && wave == owner >> 6) {
            const int at = slice * SLICE + owner * PER;
            const double w = lane < PER ? left_of(at + lane) : 0.0;
            const double cum = from_lane(base, owner & 63) + wave_prefix_f64(w, lane);
            const unsigned long long some = __ballot(w > 0.0), hit = __ballot(w > 0.0 && cum > target);
            if (lane == 0) s_pick = hit ? at + __ffsll(hit) - 1 : some ? at + 63 - __clzll(some) : -1;
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

template <typename TI, typename TO>
void launch_rows(const hs_ctx* ctx, const probs_args& p, hipStream_t st) {
    const dim3 grid(std::max(1, std::min(p.rows, ctx->n_cu * 2)));
    hipLaunchKernelGGL((probs_rows<TI, TO>), grid, dim3(1024), 0, st, p);
}

template <typename T>
void launch_verify(const verify_args& a, hipStream_t st) {
    for (int round = 0; round < a.rounds; round++)
        hipLaunchKernelGGL((verify_sums<T>), dim3(a.n_slices, a.batch), dim3(256), 0, st, a, round);
    const size_t lds = (size_t)a.n_slices * sizeof(double);
    if (lds > 48 * 1024)      // (vocabularies beyond 25 million)
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&verify_pick<T>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.batch), dim3(256), lds, st, a);
}

}  // namespace

void hs_launch_probs(const hs_ctx* ctx, const hs_probs_args* args, hipStream_t st) {
    probs_args p = {args->logits, args->out, (size_t)args->logits_stride, (size_t)args->out_stride, args->live_rows, args->rows,
                    ctx->desc.vocab, 0.f, 0.f};
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
    a.accept_len = step->accept_len; a.n_out = step->n_out; a.out_tok = step->out_tok; a.path_row = step->path_row;
    if (args->type == HS_F32) launch_verify<float>(a, st);
    else launch_verify<bf16_t>(a, st);
}
