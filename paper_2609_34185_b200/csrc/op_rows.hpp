// What the operators that take whole rows share: a row of C values in the registers of some warps, eight consecutive values to a
// lane and piece, and sums and maxima over it.
#pragma once
#include "op8.hpp"

namespace ep {

#ifdef __CUDACC__

// Eight values as they lie in memory, of 16 or 32 bits each.
template <uint32_t BITS>
struct Eight {
    uint32_t w[BITS / 4];
};
// which of a piece's eight values lie inside the row: the first n
__device__ __forceinline__ uint32_t inside(uint32_t c, uint32_t C) { return c < C ? min(8u, C - c) : 0u; }

// Values c .. c + n of a row; `vec`: the row begins on 16 bytes.  What is outside reads as zero.  KEPT: vectors that every row needs, which
// stay in L1; rows are read once.
template <uint32_t BITS, bool KEPT = false>
__device__ __forceinline__ void load_eight(const uint8_t *row, uint32_t c, uint32_t n, bool vec, Eight<BITS> &e) {
    if (vec && n == 8) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + size_t(c) * (BITS / 8));
        const uint4 a = KEPT ? __ldg(p) : __ldcs(p);
        e.w[0] = a.x, e.w[1] = a.y, e.w[2] = a.z, e.w[3] = a.w;
        if constexpr (BITS == 32) {
            const uint4 b = KEPT ? __ldg(p + 1) : __ldcs(p + 1);
            e.w[4] = b.x, e.w[5] = b.y, e.w[6] = b.z, e.w[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < BITS / 4; ++i) e.w[i] = 0;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (BITS == 32) e.w[i] = __ldcs(reinterpret_cast<const uint32_t *>(row) + c + i);
            else e.w[i / 2] |= uint32_t(__ldcs(reinterpret_cast<const uint16_t *>(row) + c + i)) << (16 * (i % 2));
        }
}
// as floats; `half`: 16-bit values are binary16, else bfloat16
template <uint32_t BITS>
__device__ __forceinline__ void to_floats(const Eight<BITS> &e, bool half, float (&v)[8]) {
    if constexpr (BITS == 32) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = __uint_as_float(e.w[i]);
    } else if (half) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[2 * i] = Fp16::lo(e.w[i]), v[2 * i + 1] = Fp16::hi(e.w[i]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[2 * i] = Bf16::lo(e.w[i]), v[2 * i + 1] = Bf16::hi(e.w[i]);
    }
}
// values c .. c + n of a row of `dtype`, rounded; `vec`: the row begins on 16 bytes
__device__ __forceinline__ void store_floats(uint8_t *row, uint32_t c, uint32_t n, int32_t dtype, bool vec, const float (&v)[8]) {
    if (dtype == EP_FP32) {
        float *p = reinterpret_cast<float *>(row) + c;
        if (vec && n == 8) {
            *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (i < n) p[i] = v[i];
        }
        return;
    }
    uint32_t w[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) w[i] = dtype == EP_FP16 ? Fp16::two(v[2 * i], v[2 * i + 1]) : Bf16::two(v[2 * i], v[2 * i + 1]);
    uint16_t *p = reinterpret_cast<uint16_t *>(row) + c;
    if (vec && n == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) p[i] = uint16_t(w[i / 2] >> (16 * (i % 2)));
}
// eight one-byte values; `vec`: the row begins on 8 bytes
__device__ __forceinline__ void store_bytes(uint8_t *row, uint32_t c, uint32_t n, bool vec, uint32_t lo, uint32_t hi) {
    if (vec && n == 8) *reinterpret_cast<uint2 *>(row + c) = make_uint2(lo, hi);
    else
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) row[c + i] = uint8_t((i < 4 ? lo : hi) >> (8 * (i % 4)));
}
// four values of at most 127.5 as INT8, the nearest, ties to even: added to 1.5 * 2^23 a float's last bits are the whole number
__device__ __forceinline__ uint32_t int8x4(float a, float b, float c, float d) {
    const float magic = 12582912.0f;
    const uint32_t ab = __byte_perm(__float_as_uint(a + magic), __float_as_uint(b + magic), 0x0040),
                   cd = __byte_perm(__float_as_uint(c + magic), __float_as_uint(d + magic), 0x0040);
    return __byte_perm(ab, cd, 0x5410);
}

// INT8 scales (ep_quantize_rows): `top` = the bits of a row's largest magnitude, in which what is not finite is the largest of all
struct Int8Scale {
    float s, inverse;             // inverse 0: the row is zeros
};
__device__ __forceinline__ Int8Scale int8_scale(uint32_t top) {
    if (top >= 0x7F800000u) return {__uint_as_float(0x7FC00000u), 0.0f};
    if (top == 0) return {1.0f, 0.0f};
    const float m = fmaxf(__uint_as_float(top), __uint_as_float(8u << 23));      // 2^-119: neither quotient leaves the normal numbers
    return {__fdiv_rn(m, 127.0f), __fdiv_rn(127.0f, m)};
}

// A sum or maximum over the row that `warps` neighbouring warps of the CTA hold; every thread of the CTA takes part.  Two buffers by turns:
// who writes one again has been through the other's barrier, and so has everybody who read it.
struct RowGroup {
    uint32_t *room;               // 2 x 32 words of shared memory
    uint32_t warps, first;        // warps of a row, the row's first one
    uint32_t turn;
    template <class T, class F>
    __device__ __forceinline__ T all(T v, F op, T none) {
#pragma unroll
        for (uint32_t m = 16; m; m >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, m));
        if (warps == 1) return v;
        const uint32_t lane = threadIdx.x & 31u;
        T *at = reinterpret_cast<T *>(room + turn);
        turn ^= 32u;
        if (lane == 0) at[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < warps ? at[first + lane] : none;
#pragma unroll
        for (uint32_t m = 16; m; m >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, m));
        return v;
    }
    __device__ __forceinline__ float sum(float v) {
        return all(v, [](float a, float b) { return a + b; }, 0.0f);
    }
    __device__ __forceinline__ uint32_t largest(uint32_t v) {
        return all(v, [](uint32_t a, uint32_t b) { return max(a, b); }, 0u);
    }
};

#endif  // __CUDACC__

}  // namespace ep
