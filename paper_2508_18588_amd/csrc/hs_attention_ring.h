// What the kernels share that walk a paged cache with tiles of 32 query rows: a row tile's state, the masks of a tile of 32 keys, the
// softmax's steps, partial and final results, and the walk through a ring of key tiles in LDS.
//
// Scores are computed transposed, S^T = K . Q^T (v_mfma_f32_32x32x16_bf16), so that a lane has the scores of one query row; the second product is
// O^T = V^T . P^T.  A is a kernel's arguments (kc, vc, hkv, hq, max_blocks, n_blocks, sinks, scale_log2, lag, part_o, part_ml, part_rows, out), S a
// sequence's span of keys: those in [0, sink_end) and from `first` on, of which L are cached; skip(kb) is where a walk that has come to kb goes on.
#pragma once
#include "hs_attention_tile.h"
#include "hs_internal.h"

namespace hs_ring {

// (a NaN stays one: the rounding alone would make an infinity of some)
__device__ __forceinline__ bf16_t to_bf16(float v) { return __builtin_isnan(v) ? (bf16_t)0x7FC0 : f32_to_bf16(v); }

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

// Sets the elements that are infinities or NaNs to 0; true if there were any.
__device__ __forceinline__ bool take_nonfinite(bf16x8& x) {
    u32x4 u = __builtin_bit_cast(u32x4, x);
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const bool lo = (u[i] & 0x7F80u) == 0x7F80u, hi = (u[i] & 0x7F800000u) == 0x7F800000u;
        any |= lo | hi;
        u[i] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
    }
    x = __builtin_bit_cast(bf16x8, u);
    return any;
}

// The pages of a tile's keys; -1: there is none, or no row sees a key of it.
struct places { int p0, p1; };

// What a row sees of a tile that not every row sees all of: bit e of the result, for key e of the lane's (two runs of eight keys).
__device__ __forceinline__ unsigned below(int n) { return (1u << min(max(n, 0), 8)) - 1u; }      // of eight keys the first n
template <int HD, typename A, typename S>
__device__ __forceinline__ unsigned seen_keys(const A& a, const S& s, const row_tile<HD>& t, const places& here, int kb, int half) {
    unsigned seen = 0;
#pragma unroll
    for (int g = 0; g < 2; g++) {
        const int base = kb + 16 * g + 8 * half, node = base - s.L;
        const unsigned old = below(t.hi - base) & (~below(t.lo - base) | below(a.sinks - base));
        // (no branches: a shift's amount is taken modulo 64)
        const uint64_t up = t.anc >> (node & 63), down = t.anc << (-node & 63);
        const unsigned nodes = (unsigned)node < 64u ? (unsigned)up : (unsigned)-node < 8u ? (unsigned)down : 0u;
        seen |= ((g ? here.p1 : here.p0) >= 0 ? (old | nodes) & 0xFFu : 0u) << (8 * g);
    }
    return seen;
}
template <typename A>
__device__ __forceinline__ bool tile_masked(const A& a, const places& here, int kb, int all_lo, int all_hi) {
    return (kb + 32 > all_hi) | ((kb < all_lo) & (kb + 32 > a.sinks)) | ((here.p0 | here.p1) < 0);
}

// Masks a tile's scores and moves the running maximum, if they exceed it by more than `lag` powers of two; returns what the sums so far are to
// be scaled by.  What the weights are relative to need not be the maximum, only near it: of a tile's 32 rows nearly always some have a new
// maximum, few a much larger one, so that with a lag of 8 the scaling, 64 products per tile, is rare (8 x 512 tokens 123 -> 113 us, 256 drafts
// 445 -> 432).  Weights up to 2^8 and their sums are as exact in the same types, but the largest is not exactly 1 any more and is rounded as the
// others are: the error against 64 bits grows from 0.0020 to 0.0023 of the result, of which its own rounding to bf16 is 0.0017.  Where one
// wavefront of four has rows (at most 32 per KV head) memory sets the pace, and there is no lag.
template <int HD, typename A, typename S>
__device__ __forceinline__ float take_scores(const A& a, const S& s, row_tile<HD>& t, f32x16& sc,
                                             const places& here, bool masked, int kb, int half) {
    constexpr int NDT = HD / 32;
    if (masked) {
        const unsigned seen = seen_keys<HD>(a, s, t, here, kb, half);
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const unsigned keep = (unsigned)((int)(seen << (31 - e)) >> 31);
            sc[e] = __uint_as_float((__float_as_uint(sc[e]) & keep) | (0xFF800000u & ~keep));      // (-inf)
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
    const float m_new = tmax > t.m + a.lag ? tmax : t.m;
    float alpha = 1.f;
    if (__any(m_new != t.m)) {
        alpha = fast_exp2(t.m - (m_new == -INFINITY ? 0.f : m_new));
        t.m = m_new;
#pragma unroll
        for (int dt = 0; dt < NDT; dt++)
#pragma unroll
            for (int e = 0; e < 16; e++) t.o[dt][e] *= alpha;
    }
    return alpha;
}
// Takes infinities and NaNs out of the values of a tile that not every row sees all of, since 0 times one of them is a NaN; true if there
// were any (see add_odd).
template <int HD>
__device__ __forceinline__ bool mask_values(value_tile<HD>& v) {
    // (an exponent of all ones and one in its last place go over into the sign's)
    unsigned some = 0;
#pragma unroll
    for (int pp = 0; pp < 2; pp++)
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++) {
            const u32x4 u = __builtin_bit_cast(u32x4, v.v[pp][dt]);
#pragma unroll
            for (int i = 0; i < 4; i++) some |= (u[i] & 0x7F807F80u) + 0x00800080u;
        }
    if (!__any((some & 0x80008000u) != 0)) return false;
    bool odd = false;
#pragma unroll
    for (int pp = 0; pp < 2; pp++)
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++) {
            odd |= take_nonfinite(v.v[pp][dt]);
            asm volatile("" : "+v"(v.v[pp][dt]));
        }
    return odd;
}
// Probabilities of a tile, as the second product's operand, and their sum.
template <int HD, typename A>
__device__ __forceinline__ void take_probabilities(const A& a, row_tile<HD>& t, const f32x16& sc, float alpha, bf16x8 (&pb)[2]) {
    const float m_safe = t.m == -INFINITY ? 0.f : t.m;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) {
        // (probabilities are rounded to bf16, the matrix instruction's type: half a step, at most 2^-8, each; their sum is not)
        const float p = fast_exp2(__builtin_fmaf(sc[e], a.scale_log2, -m_safe));
        psum += p;
        pb[e >> 3][e & 7] = (__bf16)p;
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(psum), __float_as_uint(psum), false, false);
    t.l = __builtin_fmaf(t.l, alpha, __uint_as_float(sw[0]) + __uint_as_float(sw[1]));
}
template <int HD>
__device__ __forceinline__ void take_values(row_tile<HD>& t, const value_tile<HD>& v, const bf16x8 (&pb)[2]) {
#pragma unroll
    for (int pp = 0; pp < 2; pp++)
#pragma unroll
        for (int dt = 0; dt < HD / 32; dt++)
            t.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v[pp][dt], pb[pp], t.o[dt], 0, 0, 0);
}

// Where the values of a tile that not every row sees all of held infinities or NaNs: the rows that do see them add them, element by
// element, with the weights that they have in the end.  Keys k0, ... as in walk_keys, which has left them out.
template <int HD, typename A, typename S>
__device__ __forceinline__ void add_odd(const A& a, const S& s, const int32_t* __restrict__ bt, int j, int k0, int k_end,
                                     int all_lo, int all_hi, row_tile<HD>& t, int lane) {
    const int half = lane >> 5, l32 = lane & 31;
    auto page = [&](int pos) {
        const int at = pos >> 4;
        const int p = at < a.max_blocks && pos < k_end && (pos < s.sink_end || pos + 16 > s.first) ? bt[at] : -1;
        return p < a.n_blocks ? p : -1;
    };
#pragma unroll 1
    for (int kb = k0; kb < k_end; kb = s.skip(kb + 32)) {
        const places here = {page(kb), page(kb + 16)};
        if (!tile_masked(a, here, kb, all_lo, all_hi)) continue;
        const bf16_t* kp = a.kc + ((size_t)max(l32 < 16 ? here.p0 : here.p1, 0) * a.hkv + j) * 16 * HD + page_order(l32 & 15) * HD + half * 8;
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; e++) sc[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < HD / 16; ks++)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + ks * 16), t.qf[ks], sc, 0, 0, 0);
        const unsigned seen = seen_keys<HD>(a, s, t, here, kb, half);
#pragma unroll 1
        for (int tok = 0; tok < 32; tok++) {
            const int at = ((tok >> 4) << 3) | (tok & 7), from = l32 + 32 * ((tok >> 3) & 1);
            float own = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e++) own = e == at ? sc[e] : own;
            const float p = fast_exp2(__builtin_fmaf(__shfl(own, from), a.scale_log2, t.m == -INFINITY ? 0.f : -t.m));
            const bool sees = (__shfl((int)seen, from) >> at) & 1;
            const bf16_t* src = a.vc + ((size_t)max(tok < 16 ? here.p0 : here.p1, 0) * a.hkv + j) * 16 * HD + (tok & 15) + half * 64;
#pragma unroll
            for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const float x = bf16_to_f32(src[(dt * 32 + 8 * (e >> 2) + (e & 3)) * 16]);
                    t.o[dt][e] = sees && !(fabsf(x) < INFINITY) ? t.o[dt][e] + p * x : t.o[dt][e];
                }
        }
    }
}

// A partition's result for the lane's row, as store_partial leaves it (the running maximum and sum in fp32, the normalised output in fp16),
// in pieces of 16 bytes: lanes l and l + 32, which hold dims 8 g .. 8 g + 3 and 8 g + 4 .. of a row, exchange halves, so that one has all eight
// of an even g, the other of an odd one.  (Half as many stores in the middle of the key stream as in pieces of 8 bytes.)
template <int HD, typename A>
__device__ __forceinline__ void put_partial(const A& a, const row_tile<HD>& t, int r0, int rt, int R, int G, int j, int c, int lane) {
    const int half = lane >> 5, rho = rt * 32 + (lane & 31);
    const float inv = t.l > 0.f ? 1.f / t.l : 0.f;      // a partition in which the row sees no key: all zero
    const int node = rho / G;
    const size_t prow = c * a.part_rows + (size_t)(r0 + node) * a.hq + j * G + (rho - node * G);
    _Float16* po = a.part_o + prow * HD + 8 * half;
#pragma unroll
    for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            unsigned x[4];      // (dims of g, of g + 1)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
                const f16x2 v = {(_Float16)(t.o[dt][4 * g + 2 * i] * inv), (_Float16)(t.o[dt][4 * g + 2 * i + 1] * inv)};
                x[i] = __builtin_bit_cast(unsigned, v);
            }
            // the upper half of the first operand and the lower half of the second change places
            const auto lo = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false), hi = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
            if (rho < R) *reinterpret_cast<u32x4*>(po + dt * 32 + 8 * g) = u32x4{lo[0], hi[0], lo[1], hi[1]};
        }
    if (half == 0 && rho < R) *reinterpret_cast<float2*>(a.part_ml + 2 * prow) = make_float2(t.m, t.l);
}

// The result of the lane's row.
template <int HD, typename A>
__device__ __forceinline__ void put_result(const A& a, const row_tile<HD>& t, int r0, int rt, int R, int G, int j, int lane) {
    const int half = lane >> 5, rho = rt * 32 + (lane & 31), node = rho / G;
    const float inv = t.l == 0.f ? 0.f : 1.f / t.l;
    bf16_t* po = a.out + ((size_t)(r0 + node) * a.hq + j * G + (rho - node * G)) * HD;
#pragma unroll
    for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
        for (int g4 = 0; g4 < 4; g4++) {
            if (rho >= R) break;
            u32x2 x;
            x.x = (uint32_t)to_bf16(t.o[dt][4 * g4] * inv) | ((uint32_t)to_bf16(t.o[dt][4 * g4 + 1] * inv) << 16);
            x.y = (uint32_t)to_bf16(t.o[dt][4 * g4 + 2] * inv) | ((uint32_t)to_bf16(t.o[dt][4 * g4 + 3] * inv) << 16);
            *reinterpret_cast<u32x2*>(po + dt * 32 + 8 * g4 + 4 * half) = x;
        }
}

// A draft's row tile before its first key.
template <int HD>
__device__ __forceinline__ void begin_tile(row_tile<HD>& t) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; dt++)
#pragma unroll
        for (int e = 0; e < 16; e++) t.o[dt][e] = 0.f;
    t.m = -INFINITY;
    t.l = 0.f;
}

// Keys k0, ... (k_end excluded) with four row tiles, a wavefront each: one stream of 32-key tiles through a ring in LDS that the wavefronts
// fill and read together.  The keys come from memory once for all rows, and three tiles of 16 KB are on their way at any time, which loads into
// registers have no room for.  A tile is a page's K or V^T block per wavefront, straight into LDS (the layout: sub_tile).  One barrier per
// tile: it says that the tile has landed (every wavefront has waited for its share) and that its predecessor has been read, whose place is
// refilled then.  idle: the wavefront has no rows, only its share of the tiles.
// LONG: there may be more than WIN_RUN tiles (and the rows are a chunk's, whose masks are not loaded but computed).  all_lo, all_hi: see
// walk_keys, for this wavefront's rows.  LATE: the rows are waited for when the pages' numbers are there and not before these are asked for.  Behind the last tile of every part_keys keys done(): the rows' state is complete, and starts again.
constexpr int WIN_RING = 4, WIN_RUN = 512;      // tiles in LDS; tiles whose pages are looked up at a time
template <int HD>
struct win_lds {
    unsigned char ring[WIN_RING * sub_tile<HD>::BYTES];
    int page[2 * WIN_RUN + 2];      // (a tile more is looked at than there are)
};
// Two pieces of a page's block, 1 KB apart in memory and in LDS, as load_to_lds_16_stream loads one: an instruction's constant offset counts for
// both addresses.
__device__ __forceinline__ __attribute__((always_inline)) void load_pair(const unsigned char* base, unsigned off0, unsigned off1, unsigned lds_off,
                                                                         const int add) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3 offset:%4 nt\n\tglobal_load_lds_dwordx4 %2, %3 offset:%5 nt"
                 :
                 : "s"(lds_off), "v"(off0), "v"(off1), "s"(base), "i"(add), "i"(add + 1024)
                 : "memory", "m0");
}
template <int HD, bool LONG, bool LATE = false, typename A, typename S, typename Done>
__device__ __forceinline__ void ring_keys(const A& a, const S& s, const int32_t* __restrict__ bt, int j, int k0, int k_end,
                                          int part_keys, int all_lo, int all_hi, row_tile<HD>& t, bool idle, win_lds<HD>& lds, Done done) {
    using T = sub_tile<HD>;
    constexpr int NKS = HD / 16, NDT = HD / 32, CPW = T::PAGE / 1024;   // 1 KB loads per wavefront and tile
    static_assert(WIN_RING == 4, "the wait counts below");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    // the tiles: n_low of them from k0 on, and the others from low_to on (behind the gap between sinks and window)
    const int k1 = s.first & ~31;
    const int n_low = k0 < k1 ? (min(min(s.sink_end, k1), k_end) - k0 + 31) >> 5 : 0;
    const int low_to = k0 < k1 ? k1 : k0;
    const int n_tiles = n_low + max(0, (k_end - low_to + 31) >> 5);
    auto key_of = [&](int i) { return i < n_low ? k0 + 32 * i : low_to + 32 * (i - n_low); };

    // the wavefront's share of a tile: K (is_v = 0) or V^T of its page `pg`
    const unsigned page_bytes = (unsigned)a.hkv * T::PAGE;
    const int is_v = wave & 1, pg = wave >> 1;
    const unsigned ring_off = (unsigned)(size_t)(hs_gemm_detail::lds_ptr_t)lds.ring + is_v * T::V + pg * T::PAGE;
    const unsigned char* base = reinterpret_cast<const unsigned char*>(is_v ? a.vc : a.kc) + (size_t)j * T::PAGE;
    // where in the page's block a lane's 16 bytes of the first load come from; those of load i lie 1 KB i further on, where K's permutation,
    // which is its own inverse, differs by an exclusive or
    const unsigned from = is_v ? T::v_from(lane) : T::k_at(lane / (HD / 8), lane % (HD / 8));
    const int key_row = (l32 & 16) | page_order(l32 & 15);
    auto load_keys = [&](int slot, key_tile<HD>& k) __attribute__((always_inline)) {
        int at = T::k_at(key_row, half);       // (chunk 2 ks + half: the permutation is an exclusive or, and so is 2 ks)
        asm volatile("" : "+v"(at));
        const unsigned char* tile = lds.ring + slot * T::BYTES;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) k.k[ks] = *reinterpret_cast<const bf16x8*>(tile + (at ^ (ks << 5)));
    };
    auto scores = [&](const key_tile<HD>& k) __attribute__((always_inline)) {
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; e++) sc[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.k[ks], t.qf[ks], sc, 0, 0, 0);
        return sc;
    };
    // (waited for here: inside the loop the wait would be for every load in flight)
    if constexpr (!LATE) {
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) asm volatile("" : "+v"(t.qf[ks]));
        if (!LONG) asm volatile("" : "+v"(t.anc), "+v"(t.lo));
    }

    int k_next = (k0 / part_keys + 1) * part_keys, k_first = k0, odd = 0;
    for (int t0 = 0; t0 < n_tiles; t0 += WIN_RUN) {
        const int t1 = LONG ? min(n_tiles, t0 + WIN_RUN) : n_tiles;
        __syncthreads();      // (the ring and the pages have been read)
        for (int i = tid; i < 2 * (t1 - t0); i += 256) {
            const int p0 = key_of(t0 + (i >> 1)) + 16 * (i & 1), at = p0 >> 4;
            int page = -1;
            if (at < a.max_blocks && p0 < k_end && (p0 < s.sink_end || p0 + 16 > s.first)) page = bt[at];
            lds.page[i] = page < a.n_blocks ? page : -1;
        }
        __syncthreads();
        if constexpr (LATE) {
#pragma unroll
            for (int ks = 0; ks < NKS; ks++) asm volatile("" : "+v"(t.qf[ks]));
            asm volatile("" : "+v"(t.anc));
        }
        // (read long before they are used, which is when they go to a scalar register: a trip to the LDS takes longer than the rest of a fetch)
        auto pages_of = [&](int i) __attribute__((always_inline)) { return *reinterpret_cast<const int2*>(&lds.page[2 * (i - t0)]); };
        int ahead = 0, f = t0, f_slot = 0, f_page = lds.page[pg];      // ahead: tiles asked for and not yet waited for
        auto fetch = [&]() __attribute__((always_inline)) {
            const unsigned char* src = base + (size_t)max(__builtin_amdgcn_readfirstlane(f_page), 0) * page_bytes;
            const unsigned dst = ring_off + f_slot * T::BYTES;
#pragma unroll
            for (int i = 0; i < CPW; i += 2) load_pair(src, is_v ? from : from ^ T::k_step(i), is_v ? from : from ^ T::k_step(i + 1), dst, i * 1024);
            f_slot = (f_slot + 1) & (WIN_RING - 1);
            ahead++;
            if (++f < t1) f_page = lds.page[2 * (f - t0) + pg];
        };
        // waits for the wavefront's own part of the tile at the head of what it asked for, then for everybody's
        auto landed = [&](bool take_one) __attribute__((always_inline)) {
            // (as long as there are tiles to ask for, three are on their way)
            if (f < t1) HS_WAIT_VMCNT(2 * CPW);
            else HS_WAIT_VMCNT(0);
            if (take_one) ahead--;
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        while (ahead < WIN_RING - 1 && f < t1) fetch();
        landed(!is_v);      // the first keys
        if (ahead < WIN_RING - 1 && f < t1) fetch();
        if (idle) {
            for (int i = t0; i < t1; i++) {
                landed(is_v || i + 1 < t1);
                if (ahead < WIN_RING - 1 && f < t1) fetch();
            }
            if (!LONG) return;
            continue;
        }
        // The keys run one tile ahead of the values: the next tile's first product needs nothing of this one's exponentials.
        int slot = 0;
        f32x16 sc;
        int2 pages = pages_of(t0);
        {
            key_tile<HD> k;
            load_keys(0, k);
            sc = scores(k);
        }
        for (int i = t0, kb = key_of(t0), after; i < t1; i++, kb = after) {
            landed(is_v || i + 1 < t1);      // this tile's values, the next one's keys
            if (ahead < WIN_RING - 1 && f < t1) fetch();
            after = i + 1 == n_low ? low_to : kb + 32;
            key_tile<HD> k;
            value_tile<HD> v;
            const places here = {__builtin_amdgcn_readfirstlane(pages.x), __builtin_amdgcn_readfirstlane(pages.y)};
            pages = pages_of(i + 1);
            load_keys((slot + 1) & (WIN_RING - 1), k);       // (of the last tile: of whatever lies there, not used)
            const bool masked = tile_masked(a, here, kb, all_lo, all_hi);
            const float alpha = take_scores<HD>(a, s, t, sc, here, masked, kb, half);
            // (only here: with the keys, the values and the masks at the same time the registers would not do)
#pragma unroll
            for (int pp = 0; pp < 2; pp++)
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    v.v[pp][dt] = *reinterpret_cast<const bf16x8*>(lds.ring + slot * T::BYTES + T::V + pp * T::PAGE + dt * 1024 + T::v_at(l32, half));
            if (masked) odd |= __any(mask_values<HD>(v));
            bf16x8 pb[2];
            // (the matrix unit goes to the wavefront that has products for it, 113 -> 107 us for 8 x 512 tokens, 28 heads, 1024 keys)
            __builtin_amdgcn_s_setprio(1);
            const f32x16 next = scores(k);
            take_probabilities<HD>(a, t, sc, alpha, pb);
            take_values<HD>(t, v, pb);
            __builtin_amdgcn_s_setprio(0);
            sc = next;
            slot = (slot + 1) & (WIN_RING - 1);
            if (i + 1 == n_tiles || after >= k_next) {
                if (odd) {
                    add_odd<HD>(a, s, bt, j, k_first, min(k_end, k_next), all_lo, all_hi, t, lane);
                    odd = 0;
                }
                done();
                k_next = (after / part_keys + 1) * part_keys;
                k_first = after;
            }
        }
        if (!LONG) return;
    }
}

}  // namespace hs_ring
