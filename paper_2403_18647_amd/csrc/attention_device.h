// Device-side helpers shared by the attention kernels: the cache's key blocks
// and the queries as matrix-core fragments, and the output rows.
#pragma once

#include "device.h"
#include "kernels.h"

namespace sdsat {

// K and V of one 32-key block through buffer resources over this (sequence,
// head)'s cache rows: one 32-bit lane offset per 16-key half of K and one for
// V, fragment offsets as wave-uniform constants (keeps the addresses out of
// the register budget).
template <typename T, int NDS, int NDT>
__device__ __forceinline__ void load_kv(Frag<T> (&kf)[2][NDS], Frag<T> (&vf)[NDT], __amdgpu_buffer_rsrc_t kr,
                                        __amdgpu_buffer_rsrc_t vr, int blk, int c, int g, uint32_t vsoff) {
    constexpr int DH = NDS * 32;
    constexpr uint32_t E = sizeof(T);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const uint32_t ko = ((uint32_t)(blk * 32 + 16 * kt + c) * DH + 8 * g) * E;
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds) kf[kt][ds] = buf_frag<T>(kr, ko, ds * 32 * E);
    }
    const uint32_t vo = ((uint32_t)blk * DH * 32 + c * 32 + 8 * g) * E;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) vf[dt] = buf_frag<T>(vr, vo, vsoff + dt * 16 * 32 * E);
}

// x as the matrix-core operand pair hi + lo (lo = the bf16 rounding remainder;
// float models use x itself and no second fragment).
template <typename T>
__device__ __forceinline__ void split_frag(const float (&x)[8], Frag<T>& hi, Frag<T>& lo) {
    hi = Frag<T>::from_f32(x);
    if constexpr (sizeof(T) == 2) {
        float r[8];
        const uint32_t w[4] = {hi.v.x, hi.v.y, hi.v.z, hi.v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = x[i] - bf16_to_f32((uint16_t)(w[i / 2] >> (16 * (i % 2))));
        lo = Frag<T>::from_f32(r);
    }
}

// Q fragments of the current row tile, in LDS: [hi / lo][ds][lane].  They are
// read where they are used, which keeps them out of the register budget: the
// index passes through an empty asm statement, so the compiler cannot hoist
// the reads out of the block loop (a volatile read would do the same but also
// makes it wait for every outstanding global load, the next blocks' K and V).
template <typename T>
__device__ __forceinline__ Frag<T> lds_frag(const Frag<T>* qs, int idx) {
    asm volatile("" : "+v"(idx));
    return qs[idx];
}

// Where columns d .. d + 3 of head h (d a multiple of 4) of block row m go: float
// rows, or the O GEMM's input in fragment order (the four stay in one chunk).
// The row is opaque, so that the offset is formed where this stands and not ahead
// of the block loop: held through it, it takes attn_kernel<bf16, 128, 1> past its
// 256 registers, and every launch then pays for scratch (1024 wide, 8 heads, one
// row, 300 keys: 11.0 -> 10.5 us).
template <int DH>
__device__ __forceinline__ size_t out_off(const AttnArgs& a, int b, int h, int m, int d) {
    int row = b * a.q + m;
    const int col = h * DH + d;
    asm volatile("" : "+v"(row));
    return a.out_f32 ? (size_t)row * a.ldo + col : frag_off(row, col, a.ldo, a.out_rows);
}

template <typename T>
__device__ __forceinline__ void store_out(const AttnArgs& a, size_t off, f32x4_t v) {
    if (a.out_f32) {
        float* po = reinterpret_cast<float*>(a.out) + off;   // the caller's: float-aligned
#pragma unroll
        for (int r = 0; r < 4; ++r) po[r] = v[r];
        return;
    }
    T* po = reinterpret_cast<T*>(a.out) + off;
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(po) = uint2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
    else
        *reinterpret_cast<f32x4_t*>(po) = v;
}

}  // namespace sdsat
