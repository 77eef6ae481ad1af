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

// Values c .. c + n of a row; `vec`: 2 if rows begin on 16 bytes, 1 on 8, else 0.  What is outside reads as zero.  KEPT: vectors that every row needs, or a row that is
// read again, which stay in L1; rows are read once.  (Value by value the next seven loads want the same sectors, so that rows stay there as well.)
template <uint32_t BITS, bool KEPT = false>
__device__ __forceinline__ void load_eight(const uint8_t *row, uint32_t c, uint32_t n, uint32_t vec, Eight<BITS> &e) {
    if (vec == 2 && n == 8) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + size_t(c) * (BITS / 8));
        const uint4 a = KEPT ? __ldg(p) : __ldcs(p);
        e.w[0] = a.x, e.w[1] = a.y, e.w[2] = a.z, e.w[3] = a.w;
        if constexpr (BITS == 32) {
            const uint4 b = KEPT ? __ldg(p + 1) : __ldcs(p + 1);
            e.w[4] = b.x, e.w[5] = b.y, e.w[6] = b.z, e.w[7] = b.w;
        }
        return;
    }
    if (vec == 1 && n == 8) {
        const uint2 *p = reinterpret_cast<const uint2 *>(row + size_t(c) * (BITS / 8));
#pragma unroll
        for (uint32_t i = 0; i < BITS / 8; ++i) {
            const uint2 a = KEPT ? __ldg(p + i) : __ldcs(p + i);
            e.w[2 * i] = a.x, e.w[2 * i + 1] = a.y;
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < BITS / 4; ++i) e.w[i] = 0;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (BITS == 32) {
                const uint32_t *p = reinterpret_cast<const uint32_t *>(row) + c + i;
                e.w[i] = KEPT ? __ldg(p) : *p;
            } else {
                const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + c + i;
                e.w[i / 2] |= uint32_t(KEPT ? __ldg(p) : *p) << (16 * (i % 2));
            }
        }
}
// the same from shared memory, all eight values or none
template <uint32_t BITS>
__device__ __forceinline__ void smem_eight(uint32_t at, bool there, Eight<BITS> &e) {
#pragma unroll
    for (uint32_t i = 0; i < BITS / 16; ++i) {
        const uint4 a = there ? ld_smem16(at + 16 * i) : make_uint4(0, 0, 0, 0);
        e.w[4 * i] = a.x, e.w[4 * i + 1] = a.y, e.w[4 * i + 2] = a.z, e.w[4 * i + 3] = a.w;
    }
}
// addresses on 16 bytes, whole multiples of 16 bytes
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Two floats side by side, for arithmetic on both at once.
struct Pair {
    uint64_t w;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(w) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
    __device__ __forceinline__ float2 two() const {
        float2 v;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(w));
        return v;
    }
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w));
    return r;
}
// as floats, of type E
template <class E>
__device__ __forceinline__ void to_pairs(const Eight<8 * sizeof(typename E::T)> &e, Pair (&v)[4]) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        if constexpr (sizeof(typename E::T) == 4) v[i] = Pair(__uint_as_float(e.w[2 * i]), __uint_as_float(e.w[2 * i + 1]));
        else v[i] = Pair(E::lo(e.w[i]), E::hi(e.w[i]));
    }
}
// the same where the type is known only when it runs; `half`: 16-bit values are binary16, else bfloat16
template <uint32_t BITS>
__device__ __forceinline__ void to_pairs(const Eight<BITS> &e, bool half, Pair (&v)[4]) {
    if constexpr (BITS == 32) to_pairs<Fp32>(e, v);
    else if (half) to_pairs<Fp16>(e, v);
    else to_pairs<Bf16>(e, v);
}
// the larger magnitude; NaN is the largest
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ float largest_of(const Pair (&v)[4], float top) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const float2 t = v[i].two();
        top = larger(larger(top, t.x), t.y);
    }
    return top;
}
// values c .. c + n of a row of `dtype`, rounded; `vec` as above
__device__ __forceinline__ void store_pairs(uint8_t *row, uint32_t c, uint32_t n, int32_t dtype, uint32_t vec, const Pair (&v)[4]) {
    const float2 a = v[0].two(), b = v[1].two(), d = v[2].two(), e = v[3].two();
    if (dtype == EP_FP32) {
        float *p = reinterpret_cast<float *>(row) + c;
        if (vec == 2 && n == 8) {
            *reinterpret_cast<float4 *>(p) = make_float4(a.x, a.y, b.x, b.y);
            *reinterpret_cast<float4 *>(p + 4) = make_float4(d.x, d.y, e.x, e.y);
        } else if (vec == 1 && n == 8) {
            float2 *q = reinterpret_cast<float2 *>(p);
            q[0] = a, q[1] = b, q[2] = d, q[3] = e;
        } else {
            const float f[8] = {a.x, a.y, b.x, b.y, d.x, d.y, e.x, e.y};
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (i < n) p[i] = f[i];
        }
        return;
    }
    uint32_t w[4];
    if (dtype == EP_FP16) w[0] = Fp16::two(a.x, a.y), w[1] = Fp16::two(b.x, b.y), w[2] = Fp16::two(d.x, d.y), w[3] = Fp16::two(e.x, e.y);
    else w[0] = Bf16::two(a.x, a.y), w[1] = Bf16::two(b.x, b.y), w[2] = Bf16::two(d.x, d.y), w[3] = Bf16::two(e.x, e.y);
    uint16_t *p = reinterpret_cast<uint16_t *>(row) + c;
    if (vec == 2 && n == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if (vec == 1 && n == 8) {
        uint2 *q = reinterpret_cast<uint2 *>(p);
        q[0] = make_uint2(w[0], w[1]), q[1] = make_uint2(w[2], w[3]);
    } else
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) p[i] = uint16_t(w[i / 2] >> (16 * (i % 2)));
}
// eight values to an address on 16 bytes (fp32: on 32)
template <class E>
__device__ __forceinline__ void store_eight(void *p, const Pair (&v)[4]) {
    const float2 a = v[0].two(), b = v[1].two(), c = v[2].two(), d = v[3].two();
    if constexpr (sizeof(typename E::T) == 4)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y), "f"(d.x), "f"(d.y) : "memory");
    else *static_cast<uint4 *>(p) = make_uint4(E::two(a.x, a.y), E::two(b.x, b.y), E::two(c.x, c.y), E::two(d.x, d.y));
}
// eight one-byte values; `vec`: 2 if rows begin on 8 bytes, 1 on 4, else 0
__device__ __forceinline__ void store_bytes(uint8_t *row, uint32_t c, uint32_t n, uint32_t vec, uint32_t lo, uint32_t hi) {
    if (vec == 2 && n == 8) *reinterpret_cast<uint2 *>(row + c) = make_uint2(lo, hi);
    else if (vec == 1 && n == 8) {
        *reinterpret_cast<uint32_t *>(row + c) = lo;
        *reinterpret_cast<uint32_t *>(row + c + 4) = hi;
    } else
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < n) row[c + i] = uint8_t((i < 4 ? lo : hi) >> (8 * (i % 4)));
}
// Eight values times `inverse` as INT8, the nearest, ties to even, for products of at most 127.5: added to 1.5 * 2^23 a float's last bits are the
// whole number.  (The products are taken one by one: the compiler makes one fused operation of a paired product and a paired sum, which rounds once
// where the definition rounds twice.)
__device__ __forceinline__ void to_int8(const Pair (&v)[4], float inverse, uint32_t &lo, uint32_t &hi) {
    uint32_t w[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const float2 x = v[i].two(), t = (Pair(__fmul_rn(x.x, inverse), __fmul_rn(x.y, inverse)) + Pair(12582912.0f)).two();
        w[i] = __byte_perm(__float_as_uint(t.x), __float_as_uint(t.y), 0x0040);
    }
    lo = __byte_perm(w[0], w[1], 0x5410);
    hi = __byte_perm(w[2], w[3], 0x5410);
}
// as E4M3
__device__ __forceinline__ void to_e4m3(const Pair (&v)[4], float inverse, uint32_t &lo, uint32_t &hi) {
    uint32_t w[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const float2 t = (v[i] * Pair(inverse)).two();
        w[i] = e4m3x2(t.x, t.y);
    }
    lo = w[0] | w[1] << 16;
    hi = w[2] | w[3] << 16;
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

// A sum or maximum over the row that `warps` neighbouring warps of the CTA hold; all of them take part.  Two buffers by turns: who writes one again has been
// through the other's barrier, and so has everybody who read it.
struct RowGroup {
    uint32_t *room;               // 2 x 32 words of shared memory
    uint32_t warps, first;        // warps of a row, the row's first one
    uint32_t barrier;             // the named barrier of the row's warps
    uint32_t turn;
    uint32_t lanes = 32;          // of a row that is not a whole warp's: a power of two
    template <class T, class F>
    __device__ __forceinline__ T all(T v, F op, T none) {
        if (lanes < 32) {
            for (uint32_t m = lanes >> 1; m; m >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, m));
            return v;
        }
#pragma unroll
        for (uint32_t m = 16; m; m >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, m));
        if (warps == 1) return v;
        const uint32_t lane = threadIdx.x & 31u;
        T *at = reinterpret_cast<T *>(room + turn);
        turn ^= 32u;
        if (lane == 0) at[threadIdx.x >> 5] = v;
        asm volatile("barrier.sync.aligned %0, %1;" ::"r"(barrier), "r"(warps * 32u) : "memory");
        // as many lanes as a power of two that holds the warps, side by side
        const uint32_t span = warps <= 4 ? 4u : warps <= 8 ? 8u : 32u, i = lane & (span - 1u);
        v = i < warps ? at[first + i] : none;
        if (span == 32) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16)), v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
        if (span >= 8) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
        v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
        return op(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
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
