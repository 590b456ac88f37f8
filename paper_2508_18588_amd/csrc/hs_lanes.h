// Exchanges between the lanes of a wavefront that stay out of the LDS unit, and the sums and maxima built on them.
#pragma once
#include <hip/hip_runtime.h>

// The value of lane (own ^ O), by DPP and permlane moves: a butterfly of __shfl_xor is a chain of trips through the LDS
// unit, for the sampler most of what a workgroup waits for when it sums one slice after another.
// (quad_perm 1 0 3 2 and 2 3 0 1; half-row mirror, then the quad mirrored back; a row rotated by eight; rows and halves
// swapped: the results of a swap of a register with itself are own and partner, in an order that depends on the lane)
template <int O>
__device__ __forceinline__ unsigned lane_xor(unsigned v) {
    if constexpr (O == 1) return __builtin_amdgcn_update_dpp(0u, v, 0xB1, 0xF, 0xF, true);
    else if constexpr (O == 2) return __builtin_amdgcn_update_dpp(0u, v, 0x4E, 0xF, 0xF, true);
    else if constexpr (O == 4)
        return __builtin_amdgcn_update_dpp(0u, __builtin_amdgcn_update_dpp(0u, v, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
    else if constexpr (O == 8) return __builtin_amdgcn_update_dpp(0u, v, 0x128, 0xF, 0xF, true);
    else {
        static_assert(O == 16 || O == 32, "within a wavefront");
        const auto sw = O == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (threadIdx.x & O) ? sw[0] : sw[1];
    }
}

template <int O>
__device__ __forceinline__ double lane_xor_f64(double v) {
    return __hiloint2double((int)lane_xor<O>((unsigned)__double2hiint(v)), (int)lane_xor<O>((unsigned)__double2loint(v)));
}
// Butterflies over 64 lanes (WIDTH = 32: over either half): every lane gets the result, added up in the same tree.
template <int WIDTH = 64>
__device__ __forceinline__ double wave_sum_f64(double v) {
    if constexpr (WIDTH == 64) v += lane_xor_f64<32>(v);
    v += lane_xor_f64<16>(v);
    v += lane_xor_f64<8>(v);
    v += lane_xor_f64<4>(v);
    v += lane_xor_f64<2>(v);
    return v + lane_xor_f64<1>(v);
}
template <int WIDTH = 64>
__device__ __forceinline__ float wave_max_f32(float v) {
    auto step = [&](unsigned other) { v = fmaxf(v, __uint_as_float(other)); };
    if constexpr (WIDTH == 64) step(lane_xor<32>(__float_as_uint(v)));
    step(lane_xor<16>(__float_as_uint(v)));
    step(lane_xor<8>(__float_as_uint(v)));
    step(lane_xor<4>(__float_as_uint(v)));
    step(lane_xor<2>(__float_as_uint(v)));
    step(lane_xor<1>(__float_as_uint(v)));
    return v;
}

// Workgroup barrier for values in LDS alone: unlike __syncthreads it leaves loads from memory on their way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ double block_sum_f64(double v, double* red) {
    v = wave_sum_f64(v);
    lds_barrier();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    lds_barrier();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ float block_max_f32(float v, float* red) {
    v = wave_max_f32(v);
    lds_barrier();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    lds_barrier();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// Sum over the lanes up to and including this one, in lane order by a fixed tree.
__device__ __forceinline__ double wave_prefix_f64(double v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __hiloint2double(__shfl_up(__double2hiint(v), o), __shfl_up(__double2loint(v), o));
        if (lane >= o) v += t;
    }
    return v;
}
