// Rotary positions.
#include <cmath>

#include "op_rows.hpp"

using namespace ep;

namespace {

constexpr uint32_t kTable = 4096;                // cosines and sines that a CTA holds at most
constexpr uint32_t kThreads = 256, kAtOnce = 4;  // units that a thread has under way

// ======================================================================================================================
// (u, v) -> f (u cos a - v sin a, v cos a + u sin a),   a = position * frequency[i]
//
// A far position times a frequency has more turns than 32 bits can hold beside the fraction that counts (200 000 radians in fp32 are
// off by 0.008).  So a frequency is a fraction of a turn in 64 bits, whole numbers multiply it, and what passes 64 bits are whole turns, which fall
// away by themselves: no reduction.  The step is off by 2^-64 of a turn and by 2^-52 of itself (the product and the reciprocal of 2 pi are doubles, as the
// frequency is: its own last bit makes half as much), which a position multiplies: the first by 2^-32 of a turn at 2^32, 2^-24 at 2^40.  The product's first bits go to sincospi, for 32-bit values all of them count.
// (96 bits, by a second double and a longer product, took 8192 tokens of a single head from 4.1 to 4.4 us, for positions that no context has.)
// Bound by memory: a CTA works out its tokens' cosines and sines once, for all heads (48 heads of 128 of 8192 tokens BF16 in 33.7 us, 6.0 TB/s; with
// cosines read 8 bytes at a time, 64 bytes apart, 43.7).
// ======================================================================================================================
struct RotaryParams {
    const uint8_t *x;
    uint8_t *o;
    const void *positions;
    const double *frequencies;
    int64_t ldx, ldx_head, ldo, ldo_head;        // bytes
    uint32_t T, heads, dim, pairs;
    uint32_t tokens, parts;                      // tokens of a CTA; CTAs that share these tokens' heads
    uint32_t per_head;                           // units of a head: pieces that turn (half layout: pairs of pieces), then pieces that stay
    uint32_t turning;
    uint32_t apart;                              // bytes between the two pieces of a unit that stays (0: it is one)
    uint32_t heads_of_part;
    uint32_t step_j, step_h, step_t;             // kThreads units further: units of a head, heads, tokens
    uint32_t lines;                              // tokens whose cosines the threads work out at a time
    uint64_t by_units, by_heads, by_columns;     // 2^32 / n, rounded up: n / per_head, n / heads_of_part, n / min(pairs, kThreads)
    uint32_t wide_positions;
    float factor;
};

// n / d for n < 256 and d < 2^24, of 2^32 / d rounded up (a division takes the threads longer than their first loads need to be put together)
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint64_t inverse) { return uint32_t((n * inverse) >> 32); }
inline uint64_t inverse_of(uint32_t d) { return ((uint64_t(1) << 32) + d - 1u) / d; }


__device__ __forceinline__ uint64_t turn_fraction(double radians) {
    double t = radians * 0.15915494309189533577;                                 // 1 / (2 pi)
    t -= rint(t);
    return uint64_t(__double2ll_rn(t * 18446744073709551616.0));
}
template <class E>
__device__ __forceinline__ float2 cosine_sine(int64_t position, uint64_t step, float factor) {
    const uint64_t angle = uint64_t(position) * step;                                  // of a turn, in 2^-64
    const uint32_t high = uint32_t(angle >> 32);
    float s, c;
    if constexpr (sizeof(typename E::T) == 4) {
        // The first 24 bits, the nearest, go to sincospi, exactly; what that leaves, d radians, turns the result on: 1 - d^2 / 2 is 1.  (A single
        // head of 8192 tokens 4.45 -> 4.70 us, 48 of 4096 32.3 -> 32.5.)
        const float d = float(int32_t(__funnelshift_r(uint32_t(angle), high, 8))) * 8.719671245021580e-17f;    // 2 pi / 2^56
        sincospif(float(int32_t((high + 128u) & ~255u)) * 4.656612873077393e-10f, &s, &c);                     // 2^-31: half turns
        return make_float2(fmaf(-s, d, c) * factor, fmaf(c, d, s) * factor);
    } else {
        // (32 bits, of which the float keeps 24: pi 2^-25 in a result that is rounded to 2^-11 or 2^-8.  The rest costs a single head of 200 000 tokens 8 %.)
        sincospif(float(int32_t(high)) * 4.656612873077393e-10f, &s, &c);
        return make_float2(c * factor, s * factor);
    }
}

// a piece of V values of type E: V * sizeof a power of two up to 16 bytes, read and written as one
template <class E, uint32_t V>
struct Piece {
    using T = typename E::T;
    static constexpr uint32_t kBytes = V * sizeof(T);
    uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
    __device__ __forceinline__ void load(const uint8_t *p) {
        if constexpr (kBytes == 16) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        } else if constexpr (kBytes == 8) {
            const uint2 a = *reinterpret_cast<const uint2 *>(p);
            w[0] = a.x, w[1] = a.y;
        } else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const uint32_t *>(p);
        else w[0] = *reinterpret_cast<const uint16_t *>(p);
    }
    __device__ __forceinline__ void store(uint8_t *p) const {
        if constexpr (kBytes == 16) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t *>(p) = w[0];
        else *reinterpret_cast<uint16_t *>(p) = uint16_t(w[0]);
    }
    __device__ __forceinline__ float get(uint32_t i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i % 2 ? E::hi(w[i / 2]) : E::lo(w[i / 2]);
    }
    __device__ __forceinline__ void set(const float (&v)[V]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (uint32_t i = 0; i < V; ++i) w[i] = __float_as_uint(v[i]);
        } else if constexpr (V == 1) w[0] = E::bits(E::of(v[0]));
        else {
#pragma unroll
            for (uint32_t i = 0; i < V; i += 2) w[i / 2] = E::two(v[i], v[i + 1]);
        }
    }
};

// CTAs of an SM that the registers leave room for (what a thread has under way takes 8 to 32 of them)
constexpr uint32_t ctas_of_sm(uint32_t piece, bool next) { return piece == 16 ? (next ? 4u : 3u) : piece == 8 && !next ? 4u : 5u; }

// V: values of a piece; NEXT: pairs side by side (V = 1: a unit is the two pieces of one pair in either layout)
template <class E, uint32_t V, bool NEXT>
__global__ void __launch_bounds__(kThreads, ctas_of_sm(Piece<E, V>::kBytes, NEXT)) rotary_kernel(const __grid_constant__ RotaryParams P) {
    constexpr uint32_t kSize = sizeof(typename E::T);
    constexpr bool kTwo = !NEXT || V == 1;                                      // a unit that turns is two pieces
    // A unit's cosines and sines two pairs at a time, {c, c', s, s'}, in planes: units that lie side by side read 16 bytes side by side.
    constexpr uint32_t kPairs = NEXT ? (V > 1 ? V / 2 : 1) : V;                 // of a unit
    extern __shared__ __align__(16) float table[];
    auto place = [&](uint32_t token, uint32_t i) {
        if constexpr (kPairs == 1) return 2u * (token * P.pairs + i);
        return 2u * token * P.pairs + 4u * ((i % kPairs) / 2u * P.turning + i / kPairs) + i % 2u;
    };
    op_wait_for_stream();
    const uint32_t t0 = (blockIdx.x / P.parts) * P.tokens, part = blockIdx.x % P.parts, tokens = min(P.tokens, P.T - t0);
    const uint32_t h0 = part * P.heads_of_part, heads = P.heads_of_part;
    Piece<E, V> a[kAtOnce], b[kAtOnce];
    int64_t to[kAtOnce];
    uint32_t at[kAtOnce], apart[kAtOnce];
    // Units are counted through the heads and the tokens; a thread's next one is kThreads further.
    uint32_t h = quotient(threadIdx.x, P.by_units), j = threadIdx.x - h * P.per_head, t = quotient(h, P.by_heads);
    h -= t * heads;
    auto load = [&]() {
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            at[k] = ~0u;
            apart[k] = 0;
            to[k] = -1;
            if (t < tokens) {
                uint32_t c;                                                     // the unit's first value
                if (j < P.turning) {
                    c = NEXT && V == 1 ? 2 * j : j * V;
                    at[k] = 2u * t * P.pairs + (kPairs == 1 ? 2u : 4u) * j;
                    apart[k] = kTwo ? (NEXT ? kSize : P.pairs * kSize) : 0;
                } else {
                    c = 2 * P.pairs + (j - P.turning) * V;
                    apart[k] = kTwo ? P.apart : 0;
                }
                const uint8_t *src = P.x + int64_t(t0 + t) * P.ldx + int64_t(h0 + h) * P.ldx_head + c * kSize;
                to[k] = int64_t(t0 + t) * P.ldo + int64_t(h0 + h) * P.ldo_head + c * kSize;
                a[k].load(src);
                if (kTwo && apart[k]) b[k].load(src + apart[k]);
            }
            j += P.step_j, h += P.step_h, t += P.step_t;
            if (j >= P.per_head) j -= P.per_head, ++h;
            if (h >= heads) h -= heads, ++t;
        }
    };
    load();                                                                     // (under way while the cosines are worked out)
    const uint32_t columns = min(P.pairs, kThreads), lines = P.lines, line = quotient(threadIdx.x, P.by_columns);
    auto position_of = [&](uint32_t n) {
        return P.wide_positions ? static_cast<const int64_t *>(P.positions)[t0 + n] : int64_t(static_cast<const int32_t *>(P.positions)[t0 + n]);
    };
    if (line < lines && line < tokens) {
        const int64_t first = position_of(line);                                // (asked for together with the frequency)
        for (uint32_t i = threadIdx.x - line * columns; i < P.pairs; i += kThreads) {
            const uint64_t step = turn_fraction(P.frequencies[i]);
            float2 cs = cosine_sine<E>(first, step, P.factor);
            uint32_t p = place(line, i);
            table[p] = cs.x, table[p + (kPairs == 1 ? 1 : 2)] = cs.y;
#pragma unroll 4
            for (uint32_t n = line + lines; n < tokens; n += lines) {
                cs = cosine_sine<E>(position_of(n), step, P.factor);
                p = place(n, i);
                table[p] = cs.x, table[p + (kPairs == 1 ? 1 : 2)] = cs.y;
            }
        }
    }
    __syncthreads();
    while (true) {
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            if (to[k] < 0) break;
            if (at[k] != ~0u) {
                if constexpr (kPairs == 1) {
                    const float c = table[at[k]], s = table[at[k] + 1];
                    if constexpr (kTwo) {
                        const float p = a[k].get(0), q = b[k].get(0);
                        float u[1] = {p * c - q * s}, v[1] = {q * c + p * s};
                        a[k].set(u), b[k].set(v);
                    } else {
                        const float p = a[k].get(0), q = a[k].get(1);
                        float u[2] = {p * c - q * s, q * c + p * s};
                        a[k].set(u);
                    }
                } else {
                    float u[V], v[V];
#pragma unroll
                    for (uint32_t i = 0; i < kPairs; i += 2) {
                        const float4 cs = *reinterpret_cast<const float4 *>(table + at[k] + 2u * i * P.turning);
                        if constexpr (NEXT) {
#pragma unroll
                            for (uint32_t m = 0; m < 2; ++m) {
                                const float p = a[k].get(2 * (i + m)), q = a[k].get(2 * (i + m) + 1), c = m ? cs.y : cs.x, s = m ? cs.w : cs.z;
                                u[2 * (i + m)] = p * c - q * s;
                                u[2 * (i + m) + 1] = q * c + p * s;
                            }
                        } else {
                            const Pair c(cs.x, cs.y), s(cs.z, cs.w), p(a[k].get(i), a[k].get(i + 1)), q(b[k].get(i), b[k].get(i + 1));
                            const float2 x = fma2(p, c, q * s * Pair(-1.0f)).two(), y = fma2(q, c, p * s).two();
                            u[i] = x.x, u[i + 1] = x.y, v[i] = y.x, v[i + 1] = y.y;
                        }
                    }
                    a[k].set(u);
                    if constexpr (!NEXT) b[k].set(v);
                }
            }
            a[k].store(P.o + to[k]);
            if (kTwo && apart[k]) b[k].store(P.o + to[k] + apart[k]);
        }
        if (t >= tokens) break;
        load();
    }
}

template <class E>
int launch_rotary(RotaryParams P, bool next, bool in_place, cudaStream_t st) {
    // the largest piece of which heads, halves and addresses are whole multiples
    constexpr uint32_t kSize = sizeof(typename E::T);
    const uint64_t unit = (reinterpret_cast<uintptr_t>(P.x) | reinterpret_cast<uintptr_t>(P.o) | uint64_t(P.ldx) | uint64_t(P.ldx_head) | uint64_t(P.ldo) | uint64_t(P.ldo_head) |
                           uint64_t(P.dim) * kSize | uint64_t(next ? 2 * P.pairs : P.pairs) * kSize);
    const uint32_t bytes = unit % 16 == 0 ? 16u : unit % 8 == 0 ? 8u : kSize, V = bytes / kSize;
    P.turning = next && V > 1 ? 2 * P.pairs / V : P.pairs / V;
    // what stays: two pieces to a unit as well, where there is an even number of them
    const uint32_t stay = in_place ? 0u : (P.dim - 2 * P.pairs) / V;
    const bool two = (!next || V == 1) && stay % 2 == 0 && stay;
    P.per_head = P.turning + (two ? stay / 2 : stay);
    P.apart = two ? stay / 2 * V * kSize : 0u;
    // As many tokens to a CTA as give its threads what they load at once, or fewer where the GPU has room for more CTAs
    const uint32_t sms = uint32_t(op_sms());
    if (!sms) return EP_ERR_CUDA;
    const uint64_t per_token = uint64_t(P.heads) * P.per_head;
    uint64_t tokens = kThreads * kAtOnce / per_token;
    if (tokens > kTable / P.pairs) tokens = kTable / P.pairs;
    const uint64_t spread = (uint64_t(P.T) + 2 * sms - 1) / (2 * sms);
    if (tokens > spread) tokens = spread;
    if (tokens < 1) tokens = 1;
    P.tokens = uint32_t(tokens);
    const uint64_t ctas = (uint64_t(P.T) + tokens - 1) / tokens;
    P.parts = 1;
    while (P.parts < 8 && ctas * P.parts < sms && per_token * tokens > kThreads * P.parts && P.heads % (2 * P.parts) == 0) P.parts *= 2;
    P.heads_of_part = P.heads / P.parts;
    P.step_j = kThreads % P.per_head;
    P.step_t = kThreads / P.per_head / P.heads_of_part;
    P.step_h = kThreads / P.per_head - P.step_t * P.heads_of_part;
    const uint32_t columns = P.pairs < kThreads ? P.pairs : kThreads;
    P.lines = kThreads / columns;
    P.by_units = inverse_of(P.per_head);
    P.by_heads = inverse_of(P.heads_of_part);
    P.by_columns = inverse_of(columns);
    if (ctas * P.parts > 0x7FFFFFFFu || per_token * tokens > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    auto launch = [&](auto kernel) { return op_launch(kernel, uint32_t(ctas * P.parts), kThreads, P.tokens * P.pairs * 8u, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA; };
    if constexpr (kSize == 4) {
        if (V == 4) return next ? launch(rotary_kernel<E, 4, true>) : launch(rotary_kernel<E, 4, false>);
        if (V == 2) return next ? launch(rotary_kernel<E, 2, true>) : launch(rotary_kernel<E, 2, false>);
    } else {
        if (V == 8) return next ? launch(rotary_kernel<E, 8, true>) : launch(rotary_kernel<E, 8, false>);
        if (V == 4) return next ? launch(rotary_kernel<E, 4, true>) : launch(rotary_kernel<E, 4, false>);
    }
    return next ? launch(rotary_kernel<E, 1, true>) : launch(rotary_kernel<E, 1, false>);
}

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

}  // namespace

extern "C" int ep_rotary(const ep_rotary_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_rotary_job &j = *job;
    if (j.T == 0) return EP_OK;
    const uint32_t size = j.dtype == EP_FP32 ? 4 : j.dtype == EP_BF16 || j.dtype == EP_FP16 ? 2 : 0;
    if (!j.d_x || !j.d_out || !j.d_positions || !j.d_frequencies || !size || j.heads == 0 || j.heads > 65535 || j.pairs == 0 || j.dim > 1024 || 2 * uint64_t(j.pairs) > j.dim ||
        j.T > 0x7FFFFF00u || (j.position_bits != 32 && j.position_bits != 64) || !aligned(j.d_x, size) || !aligned(j.d_out, size) ||
        !aligned(j.d_positions, uintptr_t(j.position_bits / 8)) || !aligned(j.d_frequencies, 8))
        return EP_ERR_BAD_ARG;
    const int64_t most = int64_t(1) << 40;
    for (const int64_t ld : {j.ldx, j.ldx_head, j.ldo, j.ldo_head})
        if (ld < 0 || ld >= most) return EP_ERR_BAD_ARG;
    // What is written is written once: rows lie apart and heads lie apart, and all heads of a row lie before the next row, or all rows of a head before the next head.
    if ((j.T > 1 && j.ldo < int64_t(j.dim)) || (j.heads > 1 && j.ldo_head < int64_t(j.dim))) return EP_ERR_BAD_ARG;
    if (j.T > 1 && j.heads > 1 && j.ldo < int64_t(j.heads - 1u) * j.ldo_head + int64_t(j.dim) && (j.ldo_head - int64_t(j.dim)) / j.ldo < int64_t(j.T - 1u)) return EP_ERR_BAD_ARG;
    const bool in_place = j.d_x == j.d_out;
    if (in_place && (j.ldx != j.ldo || j.ldx_head != j.ldo_head)) return EP_ERR_BAD_ARG;
    RotaryParams P;
    std::memset(&P, 0, sizeof(P));
    P.x = static_cast<const uint8_t *>(j.d_x);
    P.o = static_cast<uint8_t *>(j.d_out);
    P.positions = j.d_positions;
    P.frequencies = j.d_frequencies;
    P.ldx = j.ldx * size;
    P.ldx_head = j.ldx_head * size;
    P.ldo = j.ldo * size;
    P.ldo_head = j.ldo_head * size;
    P.T = j.T;
    P.heads = j.heads;
    P.dim = j.dim;
    P.pairs = j.pairs;
    P.wide_positions = j.position_bits == 64;
    P.factor = j.factor;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (j.dtype == EP_BF16) return launch_rotary<Bf16>(P, j.interleaved != 0, in_place, st);
    if (j.dtype == EP_FP16) return launch_rotary<Fp16>(P, j.interleaved != 0, in_place, st);
    return launch_rotary<Fp32>(P, j.interleaved != 0, in_place, st);
}

extern "C" int ep_rotary_frequencies(uint32_t pairs, double base, double stretch, double original, double fast, double slow, double *out) {
    if (!out || pairs == 0 || !(base > 0) || !(stretch >= 1) || !(original >= 0) || (original > 0 && !(fast > slow)) || !std::isfinite(base) || !std::isfinite(stretch) ||
        !std::isfinite(original))
        return EP_ERR_BAD_ARG;
    for (uint32_t i = 0; i < pairs; ++i) {
        const double f = std::pow(base, -double(i) / double(pairs));
        double k = 0.0;
        if (original > 0) {
            k = (original * f / 6.283185307179586 - slow) / (fast - slow);
            k = k < 0.0 ? 0.0 : k > 1.0 ? 1.0 : k;
        }
        out[i] = f * (k + (1.0 - k) / stretch);
        if (!std::isfinite(out[i])) return EP_ERR_BAD_ARG;                              // (of a base next to 0, of bounds that are infinite)
    }
    return EP_OK;
}
