// Norms before and after a block, fused with the block's gate and the residual, into a 16- or 32-bit type or an 8-bit container.
#include "op_rows.hpp"

using namespace ep;

namespace {

constexpr uint32_t kMaxColumns = 32768, kStreamRoom = 224 * 1024;
__device__ unsigned int g_norm_status = 0;

// ======================================================================================================================
//   b = norm(x) (o + p),   r = c h + g b,   z = norm(r) (o + w) + d,   norm(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps)
//
// A row stays in the registers of its warps from its first byte to its last: x and h are read once, r and z written once, whatever
// stands between.  Deviations from the mean are summed in a second walk through the registers, so that nothing cancels.
// Bound by memory for many rows (8192 x 5120 BF16, two norms and a residual, 60.5 us: 5.5 TB/s; 327680 x 128 32.6 us), by the launch and two to five exchanges
// between warps for few (16 x 5120 2.6 us).
// ======================================================================================================================
struct NormVector {
    const uint8_t *d;
    int64_t pitch;                // bytes between groups
    uint32_t rows;                // of a group; 0: one vector for all rows
    int32_t dtype;
    uint32_t vec;
    uint32_t kept;                // where the stream's kernel has it in shared memory
};
struct NormParams {
    const uint8_t *x, *h;
    uint8_t *r, *z, *s;
    int64_t ldx, ldh, ldr, ldz, lds;      // bytes; scales: elements
    NormVector w, d, g, p;
    float c, offset, eps, columns, inverse;      // (inverse: of columns; a mean is divided, so that a row of equal 16-bit values, whose sum is exact, has none but zeros left)
    uint32_t T, C;
    uint32_t warps, rows;         // warps of a row, rows of a CTA
    uint32_t lanes;               // of a row that takes less than a warp (32: whole warps)
    uint32_t slots, kept;         // of the stream's kernel: rows that shared memory has room for, bytes of vectors there,
    uint32_t stretch;             // rows that share their vectors (0: all)
    int32_t x_half, h_half, r_dtype, z_dtype, center;
    uint32_t x_vec, h_vec, r_vec, z_vec;
};

__device__ __forceinline__ void load_vector(const NormVector &V, uint32_t row, uint32_t c, uint32_t n, float offset, Pair (&v)[4]) {
    const uint8_t *at = V.d + int64_t(V.rows ? row / V.rows : 0) * V.pitch;
    if (V.dtype == EP_FP32) {
        Eight<32> e;
        load_eight<32, true>(at, c, n, V.vec, e);
        to_pairs<32>(e, false, v);
    } else {
        Eight<16> e;
        load_eight<16, true>(at, c, n, V.vec, e);
        to_pairs<16>(e, V.dtype == EP_FP16, v);
    }
    if (offset != 0.0f)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[j] = v[j] + Pair(offset);
}

// v becomes (v - mean) / sqrt(mean square of that + eps).  What is outside the row is zero before and after (or NaN, where all of the row is).
template <uint32_t N>
__device__ __forceinline__ void normed(const NormParams &P, RowGroup &group, const uint32_t (&n)[N], Pair (&v)[N][4]) {
    if (P.center) {
        Pair sum(0.0f);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) sum = sum + ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3]));
        const float2 two = sum.two();
        const Pair mean(-(group.sum(two.x + two.y) / P.columns));
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] + mean;
            if (n[i] < 8) {
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    const float2 t = v[i][j].two();
                    v[i][j] = Pair(2 * j < n[i] ? t.x : 0.0f, 2 * j + 1 < n[i] ? t.y : 0.0f);
                }
            }
        }
    }
    Pair squares(0.0f), more(0.0f);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
#pragma unroll
        for (uint32_t j = 0; j < 4; j += 2) squares = fma2(v[i][j], v[i][j], squares), more = fma2(v[i][j + 1], v[i][j + 1], more);
    const float2 two = (squares + more).two();
    const Pair f(rsqrtf(group.sum(two.x + two.y) * P.inverse + P.eps));          // (good to 2^-22.9; a root and two quotients take 60 instructions of some 330)
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] * f;
}

// z of a row to memory: `put(i)` is called for each piece with what it becomes; every lane takes part
template <uint32_t N, class PUT>
__device__ __forceinline__ Int8Scale int8_pieces(RowGroup &group, const Pair (&v)[N][4], PUT put) {
    float top = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) top = largest_of(v[i], top);
    const Int8Scale s = int8_scale(group.largest(__float_as_uint(top)));
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        uint32_t lo, hi;
        to_int8(v[i], s.inverse, lo, hi);
        if (s.s != s.s) lo = hi = 0;
        put(i, lo, hi);
    }
    return s;
}
template <uint32_t N, class PUT>
__device__ __forceinline__ void e4m3_pieces(const RowGroup &group, Pair (&v)[N][4], PUT put) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {                                   // a block of 128 values is sixteen lanes'
        float top = largest_of(v[i], 0.0f);
        if (__any_sync(0xFFFFFFFFu, __float_as_uint(top) >= 0x7F800000u)) {        // without what is not finite, which becomes NaN
            top = 0.0f;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                float2 t = v[i][j].two();
                if (__float_as_uint(fabsf(t.x)) >= 0x7F800000u) t.x = __uint_as_float(0x7FFFFFFFu);
                if (__float_as_uint(fabsf(t.y)) >= 0x7F800000u) t.y = __uint_as_float(0x7FFFFFFFu);
                v[i][j] = Pair(t.x, t.y);
                top = fmaxf(fmaxf(top, fabsf(t.x)), fabsf(t.y));
            }
        }
        uint32_t bits = __float_as_uint(top);
#pragma unroll
        for (uint32_t m = 1; m < 16; m <<= 1) {
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, bits, m);
            if (m < group.lanes) bits = max(bits, other);
        }
        const uint32_t e = scale_exponent(__uint_as_float(bits), 127u);
        uint32_t lo, hi;
        to_e4m3(v[i], pow2_inverse(e), lo, hi);
        put(i, lo, hi, uint8_t(e));
    }
}

// ---- any rows: straight from memory -------------------------------------------------------------------------------------------
// Any types, alignment and up to 32768 columns.  Conversions and vectors from L1 bound it where rows begin on 16 bytes (8192 x 5120 BF16 beside FP16 62.8 us, with both norms 81.7); where they
// begin anywhere, the way from L1: eight loads one after another take the same sectors (2300 x 3427 FP32 with a residual 50 us, floor 19.6, L2 brings 480 MB for 126).
template <uint32_t XBITS, uint32_t HBITS, uint32_t N, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS) norm_kernel(const __grid_constant__ NormParams P) {
    __shared__ uint32_t room[64];
    op_wait_for_stream();
    const uint32_t warp = threadIdx.x >> 5, of = P.lanes < 32 ? threadIdx.x / P.lanes : warp / P.warps;
    const uint32_t row = blockIdx.x * P.rows + of, l = threadIdx.x - of * (P.lanes < 32 ? P.lanes : P.warps * 32u), apart = P.warps * 256u;
    RowGroup group{room, P.warps, of * P.warps, 1u + of, 0, P.lanes};
    Eight<XBITS> x[N];
    Eight<HBITS> h[N];
    uint32_t n[N];
    Pair v[N][4];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t c = i * apart + l * 8u;
        n[i] = row < P.T ? inside(c, P.C) : 0u;
        load_eight<XBITS>(P.x + int64_t(row) * P.ldx, c, n[i], P.x_vec, x[i]);
        if (P.h) load_eight<HBITS>(P.h + int64_t(row) * P.ldh, c, n[i], P.h_vec, h[i]);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) to_pairs<XBITS>(x[i], P.x_half, v[i]);
    auto times = [&](const NormVector &V, float offset) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            Pair w[4];
            load_vector(V, row, i * apart + l * 8u, n[i], offset, w);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] * w[j];
        }
    };
    if (P.p.d) {
        normed<N>(P, group, n, v);
        times(P.p, P.offset);
    }
    if (P.g.d) times(P.g, 0.0f);
    if (P.h)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            Pair old[4];
            to_pairs<HBITS>(h[i], P.h_half, old);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = fma2(Pair(P.c), old[j], v[i][j]);
        }
    if (P.r)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) store_pairs(P.r + int64_t(row) * P.ldr, i * apart + l * 8u, n[i], P.r_dtype, P.r_vec, v[i]);
    normed<N>(P, group, n, v);
    if (P.w.d) times(P.w, P.offset);
    if (P.d.d)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            Pair d[4];
            load_vector(P.d, row, i * apart + l * 8u, n[i], 0.0f, d);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] + d[j];
        }
    uint8_t *z = P.z + int64_t(row) * P.ldz;
    if (P.z_dtype == EP_INT8) {
        const Int8Scale s = int8_pieces<N>(group, v, [&](uint32_t i, uint32_t lo, uint32_t hi) { store_bytes(z, i * apart + l * 8u, n[i], P.z_vec, lo, hi); });
        if (l == 0 && row < P.T) reinterpret_cast<float *>(P.s)[row] = s.s;
    } else if (P.z_dtype == EP_FP8_E4M3) {
        e4m3_pieces<N>(group, v, [&](uint32_t i, uint32_t lo, uint32_t hi, uint8_t e) {
            store_bytes(z, i * apart + l * 8u, n[i], P.z_vec, lo, hi);
            if ((l & 15u) == 0 && n[i]) P.s[int64_t(row) * P.lds + (i * apart + l * 8u) / 128u] = e;
        });
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) store_pairs(z, i * apart + l * 8u, n[i], P.z_dtype, P.z_vec, v[i]);
    }
}

// ---- few rows that begin on 16 bytes: the same, a piece to a lane, with types known -----------------------------------------------------
// (Some tens of rows wait for launch and exchanges, some hundreds for instructions: 5120 columns in 7800 of a warp's the general way.)
template <class X, class H>
__global__ void __launch_bounds__(1024) norm_few_kernel(const __grid_constant__ NormParams P) {
    constexpr uint32_t XB = sizeof(typename X::T), HB = sizeof(typename H::T);
    __shared__ uint32_t room[64];
    op_wait_for_stream();
    const uint32_t warp = threadIdx.x >> 5, of = warp / P.warps, row = blockIdx.x * P.rows + of, l = threadIdx.x - of * P.warps * 32u;
    const bool there = row < P.T && l * 8u < P.C;
    RowGroup group{room, P.warps, of * P.warps, 1u + of, 0};
    Eight<8 * XB> x;
    Eight<8 * HB> h;
    const uint32_t n[1] = {there ? 8u : 0u};
    load_eight<8 * XB>(P.x + int64_t(row) * P.ldx, l * 8u, n[0], 2, x);
    if (P.h) load_eight<8 * HB>(P.h + int64_t(row) * P.ldh, l * 8u, n[0], 2, h);
    Pair v[1][4];
    to_pairs<X>(x, v[0]);
    auto vector = [&](const NormVector &V, float offset, Pair (&w)[4]) {
        const uint8_t *at = V.d + (V.rows ? int64_t(row / V.rows) * V.pitch : 0);
        if (V.dtype == EP_FP32) {
            Eight<32> e;
            load_eight<32, true>(at, l * 8u, n[0], 2, e);
            to_pairs<Fp32>(e, w);
        } else {
            Eight<16> e;
            load_eight<16, true>(at, l * 8u, n[0], 2, e);
            to_pairs<16>(e, V.dtype == EP_FP16, w);
        }
        if (offset != 0.0f)                               // (as load_vector does: a zero keeps its sign)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) w[j] = w[j] + Pair(offset);
    };
    auto times = [&](const NormVector &V, float offset) {
        Pair w[4];
        vector(V, offset, w);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[0][j] = v[0][j] * w[j];
    };
    if (P.p.d) {
        normed<1>(P, group, n, v);
        times(P.p, P.offset);
    }
    if (P.g.d) times(P.g, 0.0f);
    if (P.h) {
        Pair old[4];
        to_pairs<H>(h, old);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[0][j] = fma2(Pair(P.c), old[j], v[0][j]);
    }
    if (P.r && there) store_eight<H>(P.r + int64_t(row) * P.ldr + l * 8u * HB, v[0]);
    normed<1>(P, group, n, v);
    if (P.w.d) times(P.w, P.offset);
    if (P.d.d) {
        Pair d[4];
        vector(P.d, 0.0f, d);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v[0][j] = v[0][j] + d[j];
    }
    uint8_t *z = P.z + int64_t(row) * P.ldz;
    if (P.z_dtype == EP_INT8) {
        const Int8Scale q = int8_pieces<1>(group, v, [&](uint32_t, uint32_t lo, uint32_t hi) {
            if (there) *reinterpret_cast<uint2 *>(z + l * 8u) = make_uint2(lo, hi);
        });
        if (l == 0 && there) reinterpret_cast<float *>(P.s)[row] = q.s;
    } else if (P.z_dtype == EP_FP8_E4M3) {
        e4m3_pieces<1>(group, v, [&](uint32_t, uint32_t lo, uint32_t hi, uint8_t e) {
            if (there) {
                *reinterpret_cast<uint2 *>(z + l * 8u) = make_uint2(lo, hi);
                if ((l & 15u) == 0) P.s[int64_t(row) * P.lds + l / 16u] = e;
            }
        });
    } else if (there) {
        if (P.z_dtype == EP_FP32) store_eight<Fp32>(z + l * 32u, v[0]);
        else if (P.z_dtype == EP_FP16) store_eight<Fp16>(z + l * 16u, v[0]);
        else store_eight<Bf16>(z + l * 16u, v[0]);
    }
}

// ---- many short rows: a part of a warp each, one after another ----------------------------------------------------------------------
// Rows of up to 256 values (the heads of queries and keys): a CTA for four of them spends its time on starting (327680 x 128 82 us).  Here a lane keeps its
// piece of the vectors in registers and has the next row's piece under way.
template <class X, class H>
__global__ void __launch_bounds__(256) norm_short_kernel(const __grid_constant__ NormParams P) {
    constexpr uint32_t XB = sizeof(typename X::T), HB = sizeof(typename H::T);
    op_wait_for_stream();
    const uint32_t of = threadIdx.x / P.lanes, l = threadIdx.x - of * P.lanes, step = gridDim.x * P.rows;
    const bool mine = l * 8u < P.C;
    RowGroup group{nullptr, 1, 0, 0, 0, P.lanes};
    Pair p[4], g[4], w[4], d[4];
    auto keep = [&](const NormVector &V, float offset, Pair (&to)[4]) {
        if (V.d) load_vector(V, 0, l * 8u, mine ? 8u : 0u, offset, to);
    };
    keep(P.p, P.offset, p), keep(P.g, 0.0f, g), keep(P.w, P.offset, w), keep(P.d, 0.0f, d);
    Eight<8 * XB> x;
    Eight<8 * HB> h;
    auto ask = [&](uint64_t row) {
        const uint32_t n = mine && row < P.T ? 8u : 0u;
        load_eight<8 * XB>(P.x + int64_t(row) * P.ldx, l * 8u, n, 2, x);
        if (P.h) load_eight<8 * HB>(P.h + int64_t(row) * P.ldh, l * 8u, n, 2, h);
    };
    ask(uint64_t(blockIdx.x) * P.rows + of);
    for (uint64_t base = uint64_t(blockIdx.x) * P.rows; base < P.T; base += step) {
        const uint64_t row = base + of;
        const bool there = mine && row < P.T;
        const uint32_t n[1] = {mine ? 8u : 0u};
        Pair v[1][4], old[4];
        to_pairs<X>(x, v[0]);
        if (P.h) to_pairs<H>(h, old);
        ask(row + step);
        auto times = [&](const Pair (&by)[4]) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[0][j] = v[0][j] * by[j];
        };
        if (P.p.d) {
            normed<1>(P, group, n, v);
            times(p);
        }
        if (P.g.d) times(g);
        if (P.h)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[0][j] = fma2(Pair(P.c), old[j], v[0][j]);
        if (P.r && there) store_eight<H>(P.r + int64_t(row) * P.ldr + l * 8u * HB, v[0]);
        normed<1>(P, group, n, v);
        if (P.w.d) times(w);
        if (P.d.d)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[0][j] = v[0][j] + d[j];
        uint8_t *z = P.z + int64_t(row) * P.ldz;
        if (P.z_dtype == EP_INT8) {
            const Int8Scale q = int8_pieces<1>(group, v, [&](uint32_t, uint32_t lo, uint32_t hi) {
                if (there) *reinterpret_cast<uint2 *>(z + l * 8u) = make_uint2(lo, hi);
            });
            if (l == 0 && there) reinterpret_cast<float *>(P.s)[row] = q.s;
        } else if (P.z_dtype == EP_FP8_E4M3) {
            e4m3_pieces<1>(group, v, [&](uint32_t, uint32_t lo, uint32_t hi, uint8_t e) {
                if (there) {
                    *reinterpret_cast<uint2 *>(z + l * 8u) = make_uint2(lo, hi);
                    if ((l & 15u) == 0) P.s[int64_t(row) * P.lds + l / 16u] = e;
                }
            });
        } else if (there) {
            if (P.z_dtype == EP_FP32) store_eight<Fp32>(z + l * 32u, v[0]);
            else if (P.z_dtype == EP_FP16) store_eight<Fp16>(z + l * 16u, v[0]);
            else store_eight<Bf16>(z + l * 16u, v[0]);
        }
    }
}

// ---- many rows: brought into shared memory ahead ----------------------------------------------------------------------------------
// A row's exchanges between its warps take longer than its bytes, so an SM works on several rows at a time, a group of warps to each, and bulk
// copies bring in the next ones meanwhile.  Vectors wait in shared memory as floats: read from L1
// and turned into floats for each row they took half of the instructions (88 us instead of 69, with paired arithmetic 60.5).  A CTA's rows follow one another; where a group of rows with vectors of its own
// ends, the CTA brings in the next one's.
constexpr uint32_t kMaxSlots = 64, kAskedLimit = 1u << 22;
constexpr uint32_t kStreamFlight = 100 * 1024;
__host__ __device__ constexpr uint32_t stream_warps() { return 28u; }

// a vector in shared memory: of 32 pieces the first four values of each, then the others, so that a warp reads 512 bytes side by side
__device__ __forceinline__ void kept_vector(uint32_t at, uint32_t piece, bool there, Pair (&v)[4]) {
    const uint32_t a = at + (piece >> 5) * 1024u + (piece & 31u) * 16u;
    Eight<32> e;
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint4 q = there ? ld_smem16(a + 512u * i) : make_uint4(0, 0, 0, 0);
        e.w[4 * i] = q.x, e.w[4 * i + 1] = q.y, e.w[4 * i + 2] = q.z, e.w[4 * i + 3] = q.w;
    }
    to_pairs<Fp32>(e, v);
}

// RAW: vectors of 16 bits wait as they lie in memory, where as floats they would leave no room for two rows
template <class X, class H, uint32_t N, bool RAW>
__global__ void __launch_bounds__(stream_warps() * 32) norm_stream_kernel(const __grid_constant__ NormParams P) {
    constexpr uint32_t XB = sizeof(typename X::T), HB = sizeof(typename H::T);
    extern __shared__ __align__(16) uint8_t stages[];
    __shared__ uint32_t room[64];
    __shared__ uint64_t bars[kMaxSlots];
    __shared__ uint32_t asked[kMaxSlots];                 // the row that a slot's last copy brings
    __shared__ uint32_t abort_word_at;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, of = warp / P.warps, l = (warp - of * P.warps) * 32u + lane, apart = P.warps * 32u;
    const uint32_t abort_word = smem_u32(&abort_word_at), bar = smem_u32(bars), asked_at = smem_u32(asked), shared = smem_u32(stages), slots = shared + P.kept;
    const uint32_t x_bytes = P.C * XB, slot = x_bytes + (P.h ? P.C * HB : 0u), pieces = P.C / 8u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < P.slots; ++i) bar_init(bar + 8 * i, 1);
        st_smem(abort_word, 0);
        bar_init_done();
    }
    __syncthreads();
    op_wait_for_stream();
    // Rows r0 .. r1 by turns to the groups, and by turns to the slots; whoever has read a row brings in the next one of its slot.
    const uint32_t r0 = uint32_t(uint64_t(P.T) * blockIdx.x / gridDim.x), r1 = uint32_t(uint64_t(P.T) * (blockIdx.x + 1u) / gridDim.x);
    auto bring = [&](uint32_t row, uint32_t s) {
        bar_expect(bar + 8 * s, slot);
        bulk_load(slots + s * slot, P.x + int64_t(row) * P.ldx, x_bytes, bar + 8 * s);
        if (P.h) bulk_load(slots + s * slot + x_bytes, P.h + int64_t(row) * P.ldh, slot - x_bytes, bar + 8 * s);
        st_smem(asked_at + 4 * s, row);
    };
    if (threadIdx.x == 0)
        for (uint32_t s = 0; s < P.slots && r0 + s < r1; ++s) bring(r0 + s, s);
    RowGroup group{room, P.warps, of * P.warps, 1u + of, 0};
    uint32_t row = r0 + of, s = of % P.slots, phase = of / P.slots & 1u;
    for (uint32_t start = r0, end; start < r1; start = end) {
        end = P.stretch ? min(r1, (start / P.stretch + 1u) * P.stretch) : r1;
        if (start != r0) __syncthreads();                 // (the last stretch's vectors are not read any more)
        auto keep = [&](const NormVector &V, float offset) {
            if (!V.d || (start != r0 && V.rows == 0)) return;
            for (uint32_t i = threadIdx.x; i < pieces; i += blockDim.x) {
                if constexpr (RAW) {
                    Eight<16> e;
                    load_eight<16, true>(V.d + int64_t(V.rows ? start / V.rows : 0) * V.pitch, i * 8u, 8, 2, e);
                    *reinterpret_cast<uint4 *>(stages + V.kept + i * 16u) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
                } else {
                    Pair v[4];
                    load_vector(V, start, i * 8u, 8, offset, v);
                    Pair *to = reinterpret_cast<Pair *>(stages + V.kept + (i >> 5) * 1024u + (i & 31u) * 16u);
                    to[0] = v[0], to[1] = v[1], to[64] = v[2], to[65] = v[3];
                }
            }
        };
        keep(P.p, P.offset);
        keep(P.g, 0.0f);
        keep(P.w, P.offset);
        keep(P.d, 0.0f);
        __syncthreads();
        for (; row < end; row += P.rows) {
            const uint32_t at = slots + s * slot;
            // Another group may have the slot's last row still before it: a barrier tells a phase only from the next one, so the row has to have been asked
            // for.  (A wait that runs out leaves wrong values and says so.)
            for (uint32_t i = 0; ld_smem(asked_at + 4 * s) != row; ++i)
                if (i == kAskedLimit || ((i & 255u) == 255u && ld_smem(abort_word))) {
                    st_smem(abort_word, 1u);
                    break;
                }
            bar_wait(bar + 8 * s, phase, abort_word);
            bool there[N];
            uint32_t n[N];
            Pair v[N][4];
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                Eight<8 * XB> x;
                there[i] = i * apart + l < pieces;
                n[i] = there[i] ? 8u : 0u;
                smem_eight<8 * XB>(at + (i * apart + l) * 8u * XB, there[i], x);
                to_pairs<X>(x, v[i]);
            }
            auto vector = [&](const NormVector &V, float offset, uint32_t i, Pair (&w)[4]) {
                if constexpr (RAW) {
                    Eight<16> e;
                    smem_eight<16>(shared + V.kept + (i * apart + l) * 16u, there[i], e);
                    to_pairs<16>(e, V.dtype == EP_FP16, w);
                    if (offset != 0.0f)
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) w[j] = w[j] + Pair(offset);
                } else kept_vector(shared + V.kept, i * apart + l, there[i], w);
            };
            auto times = [&](const NormVector &V, float offset) {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i) {
                    Pair w[4];
                    vector(V, offset, i, w);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] * w[j];
                }
            };
            if (P.p.d) {
                normed<N>(P, group, n, v);
                times(P.p, P.offset);
            }
            if (P.g.d) times(P.g, 0.0f);
            if (P.h)
#pragma unroll
                for (uint32_t i = 0; i < N; ++i) {
                    Eight<8 * HB> h;
                    Pair old[4];
                    smem_eight<8 * HB>(at + x_bytes + (i * apart + l) * 8u * HB, there[i], h);
                    to_pairs<H>(h, old);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) v[i][j] = fma2(Pair(P.c), old[j], v[i][j]);
                }
            if (P.r) {
                uint8_t *r = P.r + int64_t(row) * P.ldr + l * 8u * HB;
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (there[i]) store_eight<H>(r + i * apart * 8u * HB, v[i]);
            }
            normed<N>(P, group, n, v);
            if (l == 0 && row + P.slots < r1) bring(row + P.slots, s);           // (every warp of the row has read it: all have taken part in the exchange)
            if (P.w.d) times(P.w, P.offset);
            if (P.d.d)
#pragma unroll
                for (uint32_t i = 0; i < N; ++i) {
                    Pair d[4];
                    vector(P.d, 0.0f, i, d);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) v[i][j] = v[i][j] + d[j];
                }
            uint8_t *z = P.z + int64_t(row) * P.ldz;
            if (P.z_dtype == EP_INT8) {
                const Int8Scale q = int8_pieces<N>(group, v, [&](uint32_t i, uint32_t lo, uint32_t hi) {
                    if (there[i]) *reinterpret_cast<uint2 *>(z + (i * apart + l) * 8u) = make_uint2(lo, hi);
                });
                if (l == 0) reinterpret_cast<float *>(P.s)[row] = q.s;
            } else if (P.z_dtype == EP_FP8_E4M3) {
                e4m3_pieces<N>(group, v, [&](uint32_t i, uint32_t lo, uint32_t hi, uint8_t e) {
                    if (there[i]) {
                        *reinterpret_cast<uint2 *>(z + (i * apart + l) * 8u) = make_uint2(lo, hi);
                        if ((lane & 15u) == 0) P.s[int64_t(row) * P.lds + (i * apart + l) / 16u] = e;
                    }
                });
            } else if (P.z_dtype == EP_FP32) {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (there[i]) store_eight<Fp32>(z + (i * apart + l) * 32u, v[i]);
            } else if (P.z_dtype == EP_FP16) {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (there[i]) store_eight<Fp16>(z + (i * apart + l) * 16u, v[i]);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < N; ++i)
                    if (there[i]) store_eight<Bf16>(z + (i * apart + l) * 16u, v[i]);
            }
            for (s += P.rows; s >= P.slots; s -= P.slots) phase ^= 1u;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && ld_smem(abort_word)) {
        // nothing may land after the CTA's end: each slot's last row gets its time
        for (uint32_t i = 0; i < P.slots && r0 + i < r1; ++i) bar_drain(bar + 8 * i, ((r1 - r0 - 1u - i) / P.slots) & 1u);
        atomicOr(&g_norm_status, unsigned(kStatusWait));
    }
}

template <class X, class H, uint32_t N, bool RAW>
int launch_stream(const NormParams &P, uint32_t smem, uint32_t sms, cudaStream_t st) {
    static bool configured[64] = {};
    const auto kernel = norm_stream_kernel<X, H, N, RAW>;
    if (const int rc = op_configure(kernel, kStreamRoom, configured)) return rc;
    return op_launch(kernel, sms, P.warps * P.rows * 32u, smem, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// How the stream's kernel would work on these rows, if it would.
bool stream_shape(NormParams &P, uint32_t row, uint32_t sms, uint32_t &smem, bool &raw) {
    const uint32_t pieces = P.C / 8u;
    if (P.C % 8 || pieces <= 32 || P.T < 8u * sms) return false;
    uint32_t vectors = 0;
    bool narrow = true;
    P.stretch = 0;
    for (const NormVector *v : {&P.p, &P.g, &P.w, &P.d}) {
        if (!v->d) continue;
        ++vectors;
        narrow = narrow && v->dtype != EP_FP32;
        // stretches: rows that share all their vectors (groups' lengths that are not multiples of one another are left to the other kernel)
        if (v->rows) {
            const uint32_t a = P.stretch ? P.stretch : v->rows, lo = a < v->rows ? a : v->rows, hi = a < v->rows ? v->rows : a;
            if (hi % lo) return false;
            P.stretch = lo;
        }
    }
    // as many rows at a time as there are warps for with four pieces to a lane, and 100 KB on the way: 8192 x 5120 BF16, 5 rows at a time, 5 slots
    // 61 us, 9 slots 66; 4 rows, 8 slots 60; 3 rows, 9 slots 67
    const uint32_t span = pieces <= 64 ? 64u : 128u;     // (two pieces to a lane for rows that leave half of four's lanes over)
    P.warps = (pieces + span - 1u) / span;
    P.rows = stream_warps() / P.warps;
    if (P.warps > 1 && P.rows > 15) P.rows = 15;                                 // (named barriers: 1 .. 15)
    if (P.rows < 1 || (P.stretch && P.stretch < 2u * P.rows)) return false;
    P.slots = kStreamFlight / row;
    if (P.slots < P.rows) P.slots = P.rows;
    if (P.slots < 2) P.slots = 2;
    if (P.slots > kMaxSlots) P.slots = kMaxSlots;
    for (const bool as_they_are : {false, true}) {
        if (as_they_are && !narrow) return false;
        const uint32_t each = (pieces + 31u) / 32u * (as_they_are ? 512u : 1024u);
        if (vectors * each + 2u * row > kStreamRoom) continue;
        P.kept = 0;
        for (NormVector *v : {&P.p, &P.g, &P.w, &P.d})
            if (v->d) v->kept = P.kept, P.kept += each;
        if (P.slots > (kStreamRoom - P.kept) / row) P.slots = (kStreamRoom - P.kept) / row;
        smem = P.kept + P.slots * row;
        raw = as_they_are;
        return true;
    }
    return false;
}

template <class X, class H>
int launch_whole(NormParams P, cudaStream_t st, bool &done) {
    const uint32_t sms = uint32_t(op_sms()), pieces = P.C / 8u;
    uint32_t smem = 0;
    if (sms && P.C % 8 == 0 && pieces <= 32 && !P.p.rows && !P.g.rows && !P.w.rows && !P.d.rows) {
        P.lanes = 32;
        while (P.lanes / 2 >= pieces) P.lanes /= 2;
        P.rows = 256u / P.lanes;
        const uint32_t ctas = (P.T - 1u) / P.rows + 1u, most = 3u * sms;         // (three CTAs fit an SM)
        if (ctas > most) {
            done = true;
            return op_launch(norm_short_kernel<X, H>, most, 256, 0, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
        }
    }
    bool raw = false;
    done = sms && stream_shape(P, P.C * uint32_t(sizeof(typename X::T) + (P.h ? sizeof(typename H::T) : 0)), sms, smem, raw);
    if (done) return pieces <= 64 ? launch_stream<X, H, 2, false>(P, smem, sms, st) : raw ? launch_stream<X, H, 4, true>(P, smem, sms, st) : launch_stream<X, H, 4, false>(P, smem, sms, st);
    if (pieces > 16 && pieces <= 1024) {                 // (shorter rows share a warp the general way)
        done = true;
        P.warps = (pieces + 31u) / 32u;
        P.rows = P.warps >= 4 ? 1u : 4u / P.warps;
        return op_launch(norm_few_kernel<X, H>, (P.T - 1u) / P.rows + 1u, P.warps * P.rows * 32u, 0, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
    }
    return EP_OK;
}

template <uint32_t XBITS, uint32_t HBITS>
int launch_norm(NormParams P, cudaStream_t st) {
    const uint32_t pieces = (P.C + 7u) / 8u;
    const uint32_t each = pieces <= 1024 ? 1u : pieces <= 2048 ? 4u : 8u;
    P.warps = (pieces + 32u * each - 1u) / (32u * each);
    P.lanes = 32;
    while (P.lanes / 2 >= pieces) P.lanes /= 2;                                  // short rows: a part of a warp each
    P.rows = P.warps >= 4 ? 1u : 4u / P.warps * (32u / P.lanes);
    const uint32_t threads = P.warps * P.rows * P.lanes, grid = (P.T - 1u) / P.rows + 1u;
    const cudaError_t e = each == 1 ? op_launch(norm_kernel<XBITS, HBITS, 1, 1024>, grid, threads, 0, 1, st, P)
                        : each == 4 ? op_launch(norm_kernel<XBITS, HBITS, 4, 512>, grid, threads, 0, 1, st, P)
                                    : op_launch(norm_kernel<XBITS, HBITS, 8, 512>, grid, threads, 0, 1, st, P);
    return e == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

uint32_t bytes_of(int32_t dtype) { return dtype == EP_FP32 ? 4u : dtype == EP_BF16 || dtype == EP_FP16 ? 2u : 0u; }
bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }
// a row of `size`-byte values every ld of them: whether it is one, and whether each begins on `n` bytes
bool rows_fit(const void *p, int64_t ld, uint32_t C, uint32_t size) { return aligned(p, size) && ld >= int64_t(C) && ld < (int64_t(1) << 40); }
bool rows_begin_on(uint32_t n, const void *p, int64_t ld, uint32_t size) { return aligned(p, n) && ld * size % n == 0; }
// 2 if they begin on n bytes, 1 on half of that, else 0
uint32_t rows_vec(uint32_t n, const void *p, int64_t ld, uint32_t size) { return rows_begin_on(n, p, ld, size) ? 2u : rows_begin_on(n / 2, p, ld, size) ? 1u : 0u; }

int vector_of(const ep_vector &v, uint32_t T, uint32_t C, NormVector &out) {
    std::memset(&out, 0, sizeof(out));
    if (!v.d) return EP_OK;
    const uint32_t size = bytes_of(v.dtype);
    if (!size || v.groups == 0 || T % v.groups || !aligned(v.d, size) || (v.groups > 1 && !rows_fit(v.d, v.ld, C, size))) return EP_ERR_BAD_ARG;
    out.d = static_cast<const uint8_t *>(v.d);
    out.dtype = v.dtype;
    if (v.groups > 1) out.pitch = v.ld * size, out.rows = T / v.groups;
    out.vec = rows_vec(16, v.d, v.groups > 1 ? v.ld : 0, size);
    return EP_OK;
}

const bool registered = ep::add_status_word([] { return op_status(g_norm_status); });

}  // namespace

extern "C" int ep_norm(const ep_norm_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_norm_job &j = *job;
    if (j.T == 0) return EP_OK;
    const uint32_t xs = bytes_of(j.x_dtype), hs = bytes_of(j.residual_dtype), zs = j.z_dtype == EP_FP8_E4M3 || j.z_dtype == EP_INT8 ? 1u : bytes_of(j.z_dtype);
    const bool residual = j.d_residual || j.d_residual_out;
    if (!j.d_x || !j.d_z || j.C == 0 || j.T > 0x7FFFFF00u || !xs || !zs || (residual && !hs) || !rows_fit(j.d_x, j.ldx, j.C, xs) || !rows_fit(j.d_z, j.ldz, j.C, zs) ||
        (j.d_residual && !rows_fit(j.d_residual, j.ld_residual, j.C, hs)) || (j.d_residual_out && !rows_fit(j.d_residual_out, j.ld_residual_out, j.C, hs)))
        return EP_ERR_BAD_ARG;
    // What is written in the place of what is read: the same type and rows where they were, so that each thread writes what it has read itself.  z and r are two things.
    auto in_place = [&](const void *to, int32_t to_dtype, int64_t ldto, const void *from, int32_t dtype, int64_t ld) {
        return to != from || !to || (to_dtype == dtype && (j.T == 1 || ldto == ld));
    };
    if (!in_place(j.d_z, j.z_dtype, j.ldz, j.d_x, j.x_dtype, j.ldx) || !in_place(j.d_z, j.z_dtype, j.ldz, j.d_residual, j.residual_dtype, j.ld_residual) ||
        !in_place(j.d_residual_out, j.residual_dtype, j.ld_residual_out, j.d_x, j.x_dtype, j.ldx) ||
        !in_place(j.d_residual_out, j.residual_dtype, j.ld_residual_out, j.d_residual, j.residual_dtype, j.ld_residual) || j.d_z == j.d_residual_out)
        return EP_ERR_BAD_ARG;
    if (j.z_dtype == EP_FP8_E4M3 && (!j.d_z_scales || j.ldz_scales < int64_t((j.C + 127u) / 128u))) return EP_ERR_BAD_ARG;
    if (j.z_dtype == EP_INT8 && (!j.d_z_scales || !aligned(j.d_z_scales, 4))) return EP_ERR_BAD_ARG;
    if (j.C > kMaxColumns) return EP_ERR_UNSUPPORTED;
    NormParams P;
    std::memset(&P, 0, sizeof(P));
    int rc;
    if ((rc = vector_of(j.weight, j.T, j.C, P.w)) || (rc = vector_of(j.bias, j.T, j.C, P.d)) || (rc = vector_of(j.gate, j.T, j.C, P.g)) ||
        (rc = vector_of(j.post_weight, j.T, j.C, P.p)))
        return rc;
    P.x = static_cast<const uint8_t *>(j.d_x);
    P.h = static_cast<const uint8_t *>(j.d_residual);
    P.r = static_cast<uint8_t *>(j.d_residual_out);
    P.z = static_cast<uint8_t *>(j.d_z);
    P.s = static_cast<uint8_t *>(j.d_z_scales);
    P.ldx = j.ldx * xs;
    P.ldh = j.ld_residual * hs;
    P.ldr = j.ld_residual_out * hs;
    P.ldz = j.ldz * zs;
    P.lds = j.ldz_scales;
    P.c = j.residual_scale;
    P.offset = j.weight_offset;
    P.eps = j.eps;
    P.columns = float(j.C);
    P.inverse = 1.0f / P.columns;
    P.T = j.T;
    P.C = j.C;
    P.x_half = j.x_dtype == EP_FP16;
    P.h_half = j.residual_dtype == EP_FP16;
    P.r_dtype = j.residual_dtype;
    P.z_dtype = j.z_dtype;
    P.center = j.center != 0;
    P.x_vec = rows_vec(16, j.d_x, j.ldx, xs);
    P.h_vec = j.d_residual ? rows_vec(16, j.d_residual, j.ld_residual, hs) : 0u;
    P.r_vec = j.d_residual_out ? rows_vec(16, j.d_residual_out, j.ld_residual_out, hs) : 0u;
    P.z_vec = rows_vec(zs == 1 ? 8 : 16, j.d_z, j.ldz, zs);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // what the stream's kernel reads and writes in whole pieces: bulk copies on 16 bytes, stores of 32-bit values on 32
    bool whole = P.C % 8 == 0 && P.x_vec == 2 && (!P.h || P.h_vec == 2) && rows_begin_on(zs == 1 ? 8 : 8 * zs, j.d_z, j.ldz, zs) && (!P.r || rows_begin_on(8 * hs, j.d_residual_out, j.ld_residual_out, hs));
    for (const NormVector *v : {&P.p, &P.g, &P.w, &P.d}) whole = whole && (!v->d || v->vec == 2);
    if (whole) {
        bool done = false;
        const int32_t h = P.h || P.r ? j.residual_dtype : j.x_dtype;
        rc = EP_OK;
        if (j.x_dtype == EP_BF16 && h == EP_BF16) rc = launch_whole<Bf16, Bf16>(P, st, done);
        if (j.x_dtype == EP_BF16 && h == EP_FP32) rc = launch_whole<Bf16, Fp32>(P, st, done);
        if (j.x_dtype == EP_FP16 && h == EP_FP16) rc = launch_whole<Fp16, Fp16>(P, st, done);
        if (j.x_dtype == EP_FP16 && h == EP_FP32) rc = launch_whole<Fp16, Fp32>(P, st, done);
        if (j.x_dtype == EP_FP32 && h == EP_FP32) rc = launch_whole<Fp32, Fp32>(P, st, done);
        if (done) return rc;
    }
    if (xs == 4) return j.d_residual && hs == 4 ? launch_norm<32, 32>(P, st) : launch_norm<32, 16>(P, st);
    return j.d_residual && hs == 4 ? launch_norm<16, 32>(P, st) : launch_norm<16, 16>(P, st);
}
