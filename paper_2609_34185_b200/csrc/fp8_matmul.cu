// Rounding to E4M3 in blocks of 128 with power-of-two scales, and the matrix product of operands held that way.
#include "op8.hpp"

using namespace ep;

namespace {

constexpr uint32_t kBlock = 128;                 // columns (and rows, for weights) that share a scale
__device__ unsigned int g_matmul_status = 0;

// ======================================================================================================================
// Quantisation.  For a block with largest finite magnitude a: s = the smallest power of two with a <= 448 s, q = e4m3(x / s).
// x / s is exact (s is a power of two), so there is one rounding, E4M3's.  E4M3 has its three fraction bits at every magnitude from
// 2^-6 to 448: a scale that is not a power of two would save at most one of fifteen binades and no rounding error.  What is
// not finite becomes NaN and has no part in the scale.
// Bound by memory: each value is read once into registers, where it waits for its block's maximum.
// ======================================================================================================================
struct QuantParams {
    const void *x;
    uint8_t *q, *s;
    int64_t ldx, ldq, lds;
    uint32_t T, C, blocks;        // blocks = ceil(C / 128)
    uint32_t vec;                 // rows of x and of q begin on 16 bytes
};

// N consecutive values of a row from column c on, as floats; zeros past the row's end
template <class E>
__device__ __forceinline__ void load_values(const typename E::T *row, uint32_t c, uint32_t C, bool vec, float (&v)[16 / sizeof(typename E::T)]) {
    constexpr uint32_t N = 16 / sizeof(typename E::T);
    if (vec && c + N <= C) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(row + c));
        if constexpr (N == 4) {
            v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
        } else {
            v[0] = E::lo(w.x), v[1] = E::hi(w.x), v[2] = E::lo(w.y), v[3] = E::hi(w.y);
            v[4] = E::lo(w.z), v[5] = E::hi(w.z), v[6] = E::lo(w.w), v[7] = E::hi(w.w);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] = c + i < C ? E::to(row[c + i]) : 0.0f;
    }
}
template <uint32_t N>
__device__ __forceinline__ float largest(const float (&v)[N]) {              // NaN has no part in it, infinity has
    float a = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) a = fmaxf(a, fabsf(v[i]));
    return a;
}
template <uint32_t N>
__device__ __forceinline__ void only_finite(float (&v)[N]) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
        if (!(fabsf(v[i]) < __uint_as_float(0x7F800000u))) v[i] = __uint_as_float(0x7FFFFFFFu);
}
// N of 4, 8 or 16 values; `vec`: the place is aligned to N bytes
template <uint32_t N>
__device__ __forceinline__ void store_values(uint8_t *row, uint32_t c, uint32_t C, bool vec, const float (&v)[N], float inverse) {
    uint32_t w[N / 4];
#pragma unroll
    for (uint32_t i = 0; i < N / 4; ++i)
        w[i] = e4m3x2(v[4 * i] * inverse, v[4 * i + 1] * inverse) | e4m3x2(v[4 * i + 2] * inverse, v[4 * i + 3] * inverse) << 16;
    if (vec && c + N <= C) {
        if constexpr (N == 16) *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (N == 8) *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(row + c) = w[0];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
            if (c + i < C) row[c + i] = uint8_t(w[i / 4] >> (8 * (i % 4)));
    }
}

// One scale per row and 128 columns.  A lane takes 32 bytes, so that a block of 16-bit values is eight lanes' (three
// exchanges for its maximum instead of four); a warp takes LOADS such pieces, counted through the rows.  Magnitudes are compared as
// integers, two 16-bit ones at a time.
template <class E, uint32_t LOADS>
__global__ void __launch_bounds__(128) quantize_rows_kernel(const __grid_constant__ QuantParams P) {
    using T = typename E::T;
    constexpr uint32_t N = 32 / sizeof(T), kLanes = kBlock / N, kSpan = 32 * N;
    op_wait_for_stream();
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t spans = (P.C + kSpan - 1u) / kSpan;
    uint64_t unit = (uint64_t(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5)) * LOADS;
    uint32_t t0 = uint32_t(unit / spans), s0 = uint32_t(unit - uint64_t(t0) * spans);
    uint32_t w[LOADS][8], row[LOADS], col[LOADS];
#pragma unroll
    for (uint32_t i = 0; i < LOADS; ++i) {
        row[i] = t0, col[i] = s0 * kSpan + lane * N;
        if (++s0 == spans) s0 = 0, ++t0;
        const T *src = static_cast<const T *>(P.x) + int64_t(row[i]) * P.ldx;
        if (row[i] < P.T && P.vec && col[i] + N <= P.C) {
            const uint4 lo = __ldcs(reinterpret_cast<const uint4 *>(src + col[i])), hi = __ldcs(reinterpret_cast<const uint4 *>(src + col[i]) + 1);
            w[i][0] = lo.x, w[i][1] = lo.y, w[i][2] = lo.z, w[i][3] = lo.w, w[i][4] = hi.x, w[i][5] = hi.y, w[i][6] = hi.z, w[i][7] = hi.w;
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                w[i][j] = 0;
#pragma unroll
                for (uint32_t k = 0; k < 4 / sizeof(T); ++k) {
                    const uint32_t c = col[i] + j * (4 / sizeof(T)) + k;
                    if (row[i] < P.T && c < P.C) w[i][j] |= E::bits(src[c]) << (16 * k);
                }
            }
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < LOADS; ++i) {
        // the largest magnitude's bits; what is not finite is the largest of all
        uint32_t a;
        if constexpr (N == 16) {
            a = w[i][0] & 0x7FFF7FFFu;
#pragma unroll
            for (uint32_t j = 1; j < 8; ++j) a = __vmaxu2(a, w[i][j] & 0x7FFF7FFFu);
#pragma unroll
            for (uint32_t m = 1; m < kLanes; m <<= 1) a = __vmaxu2(a, __shfl_xor_sync(0xFFFFFFFFu, a, m));
            a = max(a & 0xFFFFu, a >> 16);
        } else {
            a = w[i][0] & 0x7FFFFFFFu;
#pragma unroll
            for (uint32_t j = 1; j < 8; ++j) a = max(a, w[i][j] & 0x7FFFFFFFu);
#pragma unroll
            for (uint32_t m = 1; m < kLanes; m <<= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, m));
        }
        float top = E::of_bits(a);
        float v[N];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            if constexpr (N == 16) v[2 * j] = E::lo(w[i][j]), v[2 * j + 1] = E::hi(w[i][j]);
            else v[j] = __uint_as_float(w[i][j]);
        }
        if (__any_sync(0xFFFFFFFFu, !(top < __uint_as_float(0x7F800000u)))) {     // without what is not finite
            only_finite(v);
            top = largest(v);
#pragma unroll
            for (uint32_t m = 1; m < kLanes; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
        }
        const uint32_t e = scale_exponent(top, 127u);
        if (row[i] >= P.T) continue;
        store_values(P.q + int64_t(row[i]) * P.ldq, col[i], P.C, P.vec, v, pow2_inverse(e));
        if (col[i] < P.C && (lane & (kLanes - 1u)) == 0) P.s[int64_t(row[i]) * P.lds + col[i] / kBlock] = uint8_t(e);
    }
}

// one scale per 128 rows and 128 columns: a CTA of eight warps holds the block in registers, sixteen rows per warp
template <class E>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const __grid_constant__ QuantParams P) {
    using T = typename E::T;
    constexpr uint32_t N = 16 / sizeof(T), kLanes = kBlock / N, kRowsPerLoad = 32 / kLanes, kLoads = 16 / kRowsPerLoad;
    __shared__ float largest_of[8];
    op_wait_for_stream();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t rb = blockIdx.x / P.blocks, cb = blockIdx.x % P.blocks;
    const uint32_t t0 = rb * kBlock + warp * 16u + lane / kLanes, c = cb * kBlock + (lane % kLanes) * N;
    float v[kLoads][N];
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t t = t0 + i * kRowsPerLoad;
        if (t < P.T) load_values<E>(static_cast<const T *>(P.x) + int64_t(t) * P.ldx, c, P.C, P.vec, v[i]);
        else
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) v[i][j] = 0.0f;
    }
    auto block_max = [&]() {
        float a = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) a = fmaxf(a, largest(v[i]));
        a = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a)));      // magnitudes order like their bits
        if (lane == 0) largest_of[warp] = a;
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) a = fmaxf(a, largest_of[i]);
        return a;
    };
    float a = block_max();
    if (!(a < __uint_as_float(0x7F800000u))) {                                        // the same for the whole CTA
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) only_finite(v[i]);
        __syncthreads();
        a = block_max();
    }
    const uint32_t e = scale_exponent(a, 127u);
    const float inverse = pow2_inverse(e);
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t t = t0 + i * kRowsPerLoad;
        if (t < P.T) store_values(P.q + int64_t(t) * P.ldq, c, P.C, P.vec, v[i], inverse);
    }
    if (threadIdx.x == 0) P.s[int64_t(rb) * P.lds + cb] = uint8_t(e);
}

template <class E>
int launch_quantize(const QuantParams &P, uint32_t block_rows, cudaStream_t st) {
    cudaError_t e;
    if (block_rows == 1) {
        constexpr uint32_t kSpan = 32u * (32u / sizeof(typename E::T));
        const uint64_t pieces = uint64_t(P.T) * ((P.C + kSpan - 1u) / kSpan);
        // one piece per warp while that does not fill the GPU (4096 warps are seven for each scheduler)
        const bool few = pieces <= 4096;
        const uint64_t grid = (pieces + (few ? 3u : 15u)) / (few ? 4u : 16u);
        if (grid > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
        e = few ? op_launch(quantize_rows_kernel<E, 1>, uint32_t(grid), 128, 0, 1, st, P) : op_launch(quantize_rows_kernel<E, 4>, uint32_t(grid), 128, 0, 1, st, P);
    } else {
        const uint64_t grid = (uint64_t(P.T) + kBlock - 1u) / kBlock * P.blocks;
        if (grid > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
        e = op_launch(quantize_blocks_kernel<E>, uint32_t(grid), 256, 0, 1, st, P);
    }
    return e == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// ======================================================================================================================
// y[t, r] = a[r] sum_k (sx[t, k / 128] xq[t, k]) (sw[r / 128, k / 128] wq[r, k])
//
// On the tensor cores as D = A B^T with A = 128 rows of the weight (so that a single token still fills the instruction's 128
// lanes) and B = up to BN tokens: tcgen05.mma kind::mxf8f6f4 with one E8M0 scale for each row and 32 columns of both operands.
// A block of 128 columns takes four instructions whose four scales are the same byte; four blocks' bytes make up the word
// that tensor memory holds for a row, and the instruction's scale index picks the block's.  The products of two E4M3 numbers and the
// scales are exact, sums are held in fp32 in tensor memory.
// ======================================================================================================================
struct MatmulParams {
    const uint8_t *sx, *sw;       // sw may be null: ones
    const float *a;               // may be null: ones
    void *y;
    int64_t ldsx, ldsw, ldy;
    uint32_t T, R, blocks;        // blocks = ceil(C / 128)
    uint32_t tiles_r;             // tiles of 128 rows of the weight; a grid walks them first
    uint32_t split;               // CTAs (one cluster) that share a tile's columns
};

// 32 rows of 16 bytes without swizzle: eight rows, 128 bytes, are a unit
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {
    return uint64_t((addr >> 4) & 0x3FFFu) | (uint64_t(1) << 16) | (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t addr, uint32_t lead) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(tmem), "l"(scales_desc(addr)), "r"(lead) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "r"(lead) : "memory");
}
// E4M3 x E4M3, both K-major, E8M0 scales, M = 128, N = n; `word` = which byte of the scale words
__host__ __device__ constexpr uint32_t scaled_idesc(uint32_t n, uint32_t word) {
    return (word << 4) | ((n >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24) | (word << 29);
}

// ---- one tile per CTA, its columns shared by a cluster --------------------------------------------------------------
// Few tokens: the weight's bytes bound it, so every SM has to have some tens of KB of them in flight.  A cluster of up to
// eight CTAs takes a tile of 128 rows, each a share of the columns; at the end the CTAs lay their fp32 tiles down in shared memory and
// each adds up its share of the tokens over the cluster in rank order - no workspace, no atomics, the same bits every time.
template <uint32_t BN>
struct SplitShape {
    static constexpr uint32_t kStages = BN <= 32 ? 5 : BN == 64 ? 4 : 3;
    static constexpr uint32_t kA = kBlock * 128, kB = BN * 128, kStage = kA + kB;
    static constexpr uint32_t kSlots = 4;                                             // scale words of four blocks each
    static constexpr uint32_t kSlot = 512 + 512 * ((BN + 127) / 128);
    static constexpr uint32_t kScales = kStages * kStage, kBars = kScales + kSlots * kSlot, kSmem = kBars + 256 + 1024;
    static constexpr uint32_t kAcc = BN < 32 ? 32 : BN, kSlotCols = 4 + 4 * ((BN + 127) / 128);
    static constexpr uint32_t kCols = kAcc + kSlots * kSlotCols <= 64 ? 64 : kAcc + kSlots * kSlotCols <= 128 ? 128 : 256;
    static_assert(kAcc + kSlots * kSlotCols <= kCols && 128 * BN * 4 <= kScales);
};

template <uint32_t BN, class E>
__global__ void __launch_bounds__(128) matmul_split_kernel(const __grid_constant__ MatmulParams P, const __grid_constant__ CUtensorMap w_map,
                                                           const __grid_constant__ CUtensorMap x_map) {
    using G = SplitShape<BN>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t full = base + G::kBars, empty = full + 8 * G::kStages, sfull = empty + 8 * G::kStages, sempty = sfull + 8 * G::kSlots,
                   done = sempty + 8 * G::kSlots, slot_addr = done + 8, abort_word = slot_addr + 4;
    if (tid == 0) {
        for (uint32_t i = 0; i < G::kStages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (uint32_t i = 0; i < G::kSlots; ++i) bar_init(sfull + 8 * i, 64), bar_init(sempty + 8 * i, 1);
        bar_init(done, 1);
        st_smem(abort_word, 0);
        bar_init_done();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(G::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    op_wait_for_stream();
    const uint32_t tmem = ld_smem(slot_addr), sf = tmem + G::kAcc;
    const uint32_t tile = blockIdx.x / P.split, rank = blockIdx.x % P.split;
    const uint32_t r0 = (tile % P.tiles_r) * kBlock, t0 = (tile / P.tiles_r) * BN;
    const uint32_t kb0 = uint32_t(uint64_t(P.blocks) * rank / P.split), kb1 = uint32_t(uint64_t(P.blocks) * (rank + 1) / P.split), nk = kb1 - kb0;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t k = 0;
            for (; k < nk; ++k) {
                const uint32_t s = k % G::kStages, at = base + s * G::kStage;
                if (k >= G::kStages && !bar_wait(empty + 8 * s, (k / G::kStages - 1u) & 1u, abort_word)) break;
                bar_expect(full + 8 * s, G::kStage);
                tma_load_2d(at, &w_map, int32_t((kb0 + k) * 128u), int32_t(r0), full + 8 * s);
                tma_load_2d(at + G::kA, &x_map, int32_t((kb0 + k) * 128u), int32_t(t0), full + 8 * s);
            }
            if (ld_smem(abort_word))                     // nothing may land after the CTA's end
                for (uint32_t j = k > G::kStages ? k - G::kStages : 0; j < k; ++j) bar_drain(full + 8 * (j % G::kStages), (j / G::kStages) & 1u);
        }
    } else if (warp == 1) {
        {
            const uint32_t lead = elected();
            bool ok = true;
            for (uint32_t k = 0; k < nk && ok; ++k) {
                const uint32_t s = k % G::kStages, chunk = k / 4, slot = chunk % G::kSlots, sa = sf + slot * G::kSlotCols, sb = sa + 4;
                if (k % 4 == 0) {
                    ok = bar_wait_warp(sfull + 8 * slot, (chunk / G::kSlots) & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    const uint32_t at = base + G::kScales + slot * G::kSlot;
                    copy_scales(sa, at, lead);
#pragma unroll
                    for (uint32_t n = 0; n < (BN + 127) / 128; ++n) copy_scales(sb + 4 * n, at + 512 + 512 * n, lead);
                }
                ok = bar_wait_warp(full + 8 * s, (k / G::kStages) & 1u, abort_word);
                if (!ok) break;
                tc_after();
                const uint64_t da = operand_desc(base + s * G::kStage), db = operand_desc(base + s * G::kStage + G::kA);
                const uint32_t idesc = scaled_idesc(BN, k % 4);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) mma_scaled(tmem, da + 2 * i, db + 2 * i, idesc, sa, sb, (k | i) ? 1u : 0u, lead);
                tc_commit(empty + 8 * s, lead);
                if (k % 4 == 3) tc_commit(sempty + 8 * slot, lead);
            }
            tc_commit(done, lead);
        }
    } else {
        // the scale words: byte i of a word is the scale of block 4 chunk + i; row r of 128 lies at 16 (r % 32) + 4 (r / 32)
        const uint32_t l = tid - 64u;
        for (uint32_t chunk = 0; 4 * chunk < nk; ++chunk) {
            const uint32_t slot = chunk % G::kSlots, at = base + G::kScales + slot * G::kSlot, kb = kb0 + 4 * chunk, n = min(4u, nk - 4 * chunk);
            if (chunk >= G::kSlots && !bar_wait(sempty + 8 * slot, (chunk / G::kSlots - 1u) & 1u, abort_word)) break;
            uint32_t word = 0x7F7F7F7Fu;
            if (P.sw) {
                const uint8_t *p = P.sw + int64_t(r0 / kBlock) * P.ldsw + kb;
                word = 0;
                for (uint32_t i = 0; i < n; ++i) word |= uint32_t(__ldg(p + i)) << (8 * i);
            }
            for (uint32_t i = l; i < 128; i += 64) st_smem(at + 4 * i, word);
            for (uint32_t t = l; t < (BN + 31u) / 32u * 32u; t += 64) {
                uint32_t w = 0x7F7F7F7Fu;
                if (t < BN && t0 + t < P.T) {
                    const uint8_t *p = P.sx + int64_t(t0 + t) * P.ldsx + kb;
                    w = 0;
                    for (uint32_t i = 0; i < n; ++i) w |= uint32_t(__ldg(p + i)) << (8 * i);
                }
                st_smem(at + 512 + 512 * (t / 128) + 16 * (t % 32) + 4 * (t % 128 / 32), w);
            }
            fence_proxy_async();
            bar_arrive(sfull + 8 * slot);
        }
    }
    __syncwarp();
    bar_wait(done, 0, abort_word);
    if (ld_smem(abort_word)) bar_drain(done, 0);         // instructions in flight still read the stages
    tc_after();

    // lane = row of the weight, register = token
    const uint32_t r = r0 + warp * 32u + lane;
    const float a = P.a && r < P.R ? __ldg(P.a + r) : 1.0f;
    T *y = static_cast<T *>(P.y) + r;
    if (P.split == 1) {
#pragma unroll
        for (uint32_t c = 0; c < BN; c += 16) {
            if (t0 + c >= P.T) break;
            uint32_t v[16];
            tc_load16(tmem + ((warp * 32u) << 16) + c, v);
            tc_loaded();
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (r < P.R && t0 + c + i < P.T) y[int64_t(t0 + c + i) * P.ldy] = E::of(__uint_as_float(v[i]) * a);
        }
    } else {
        __syncthreads();                                 // (the stages are read no more: every thread has passed `done`)
#pragma unroll
        for (uint32_t c = 0; c < BN; c += 16) {
            uint32_t v[16];
            tc_load16(tmem + ((warp * 32u) << 16) + c, v);
            tc_loaded();
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) st_smem(base + ((c + i) * 128u + tid) * 4u, v[i]);
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        // this CTA's tokens, one to a warp, four rows to a lane; all CTAs' parts asked for at once, added in order
        const uint32_t c0 = BN * rank / P.split, c1 = BN * (rank + 1) / P.split, r4 = r0 + 4u * lane;
        uint32_t peer[8];
        float a4[4];
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer[p]) : "r"(base), "r"(min(p, P.split - 1u)));
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) a4[j] = P.a && r4 + j < P.R ? __ldg(P.a + r4 + j) : 1.0f;
#pragma unroll 2
        for (uint32_t c = c0 + warp; c < c1; c += 4) {
            if (t0 + c >= P.T) break;
            float4 v[8];
#pragma unroll
            for (uint32_t p = 0; p < 8; ++p)
                if (p < P.split)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w) : "r"(peer[p] + (c * 128u + 4u * lane) * 4u) : "memory");
            float sum[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (uint32_t p = 1; p < 8; ++p)
                if (p < P.split) sum[0] += v[p].x, sum[1] += v[p].y, sum[2] += v[p].z, sum[3] += v[p].w;
            T *dst = static_cast<T *>(P.y) + int64_t(t0 + c) * P.ldy + r4;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (r4 + j < P.R) dst[j] = E::of(sum[j] * a4[j]);
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_matmul_status, unsigned(kStatusWait));
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kCols) : "memory");
}

template <uint32_t BN, class E>
int launch_split(MatmulParams P, const void *x, int64_t ldx, const void *w, int64_t ldw, uint32_t C, cudaStream_t st) {
    using G = SplitShape<BN>;
    static bool configured[64] = {};
    int rc = op_configure(matmul_split_kernel<BN, E>, G::kSmem, configured);
    if (rc) return rc;
    const int sms = op_sms();
    if (sms <= 0) return EP_ERR_CUDA;
    CUtensorMap wm, xm;
    if ((rc = byte_map(&wm, w, C, P.R, uint64_t(ldw), 128, 128, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    if ((rc = byte_map(&xm, x, C, P.T, uint64_t(ldx), 128, BN, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    const uint64_t tiles = uint64_t(P.tiles_r) * ((P.T + BN - 1u) / BN);
    // Two CTAs fit an SM: as many as that allows share a tile, but none has fewer than two blocks of columns.  (Five to seven are not
    // taken: clusters of those sizes leave SMs of a GPC unused, 5120 x 17408 by one token in sevens 23.0 us, in fours 18.1.)
    P.split = 1;
    for (const uint32_t n : {2u, 3u, 4u, 8u})
        if (tiles * n <= uint64_t(2 * sms) && 2u * n <= P.blocks) P.split = n;
    if (tiles * P.split > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    return op_launch(matmul_split_kernel<BN, E>, uint32_t(tiles * P.split), 128, G::kSmem, P.split, st, P, wm, xm) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// ---- many tokens: a pair of CTAs per tile -----------------------------------------------------------------------------------
// Two CTAs share tiles of 256 rows of the weight by 192 tokens (tcgen05 cta_group::2): each has half of the weight's rows and half of the
// tokens in its shared memory, and keeps the sums of its 128 rows with all tokens in its tensor memory, twice, so that a tile is read out while the
// next one is summed.  What bounds one CTA per tile of 128 x 128 is the operands' way from L2: 8.6 GB for 8192^3, 15.6 TB/s in
// 551 us; a pair moves 5.0 GB.  (256 tokens would move 4.3, but two such accumulators leave tensor memory no room for scales.)
//   warp 0        brings the operands in, seven stages of 128 columns
//   warp 1        of the first CTA issues the products
//   warps 2, 3    scales, four blocks of columns at a time: this CTA's rows' and all tokens'
//   warps 4 - 7   sums to y
struct PairShape {
    static constexpr uint32_t kN = 192, kStages = 7, kA = kBlock * 128, kB = kN / 2 * 128, kStage = kA + kB;
    static constexpr uint32_t kSlots = 4, kSlot = 512 + 1024, kSlotCols = 12;
    static constexpr uint32_t kScales = kStages * kStage, kBars = kScales + kSlots * kSlot, kSmem = kBars + 512 + 1024;
    static constexpr uint32_t kSf = 2 * kN;                              // columns of the accumulators
    static_assert(kSf + kSlots * kSlotCols <= 512 && kSmem <= 232448);
};
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
                 "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "r"(lead) : "memory");
}
__device__ __forceinline__ void pair_copy_scales(uint32_t tmem, uint32_t addr, uint32_t lead) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
                 ::"r"(tmem), "l"(scales_desc(addr)), "r"(lead) : "memory");
}

template <class E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(256, 1)
    matmul_pair_kernel(const __grid_constant__ MatmulParams P, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map) {
    using G = PairShape;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t rank = blockIdx.x & 1u, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t full = base + G::kBars, empty = full + 8 * G::kStages, sfull = empty + 8 * G::kStages,
                   sempty = sfull + 8 * G::kSlots, acc_full = sempty + 8 * G::kSlots, acc_empty = acc_full + 16, done = acc_empty + 16, slot_addr = done + 8,
                   abort_word = slot_addr + 4;
    if (tid == 0) {
        for (uint32_t i = 0; i < G::kStages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (uint32_t i = 0; i < G::kSlots; ++i) bar_init(sfull + 8 * i, 2), bar_init(sempty + 8 * i, 1);
        for (uint32_t i = 0; i < 2; ++i) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, 8);
        bar_init(done, 1);
        st_smem(abort_word, 0);
        bar_init_done();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_sync();                                       // the other CTA's barriers are there
    tc_after();
    op_wait_for_stream();
    const uint32_t tmem = ld_smem(slot_addr);
    const uint32_t tiles = P.tiles_r * ((P.T + G::kN - 1u) / G::kN), nk = P.blocks;
    uint32_t k_all = 0, c_all = 0, n = 0;                 // blocks, words of scales and tiles so far
    bool ok = true;

    if (warp == 0) {
        for (uint32_t tile = pair; tile < tiles && ok; tile += pairs) {
            const uint32_t r0 = (tile % P.tiles_r) * 256u + rank * 128u, t0 = (tile / P.tiles_r) * G::kN + rank * (G::kN / 2);
            for (uint32_t k = 0; k < nk; ++k, ++k_all) {
                const uint32_t s = k_all % G::kStages, at = base + s * G::kStage;
                if (k_all >= G::kStages) ok = bar_wait_warp(empty + 8 * s, (k_all / G::kStages - 1u) & 1u, abort_word);
                if (!ok) break;
                if (lane == 0) {
                    if (rank == 0) bar_expect(full + 8 * s, 2 * G::kStage);       // both CTAs' halves
                    pair_load_2d(at, &w_map, int32_t(k * 128u), int32_t(r0), full + 8 * s);
                    pair_load_2d(at + G::kA, &x_map, int32_t(k * 128u), int32_t(t0), full + 8 * s);
                }
            }
        }
        // nothing may land after the pair's end (the second CTA's loads report to the first one, which waits for both)
        if (ld_smem(abort_word) && lane == 0)
            for (uint32_t j = k_all > G::kStages ? k_all - G::kStages : 0; j < k_all; ++j) bar_drain(full + 8 * (j % G::kStages), (j / G::kStages) & 1u);
    } else if (warp == 1 && rank == 0) {
        const uint32_t lead = elected();
        for (uint32_t tile = pair; tile < tiles && ok; tile += pairs, ++n) {
            const uint32_t acc = tmem + (n & 1u) * G::kN;
            if (n > 1u) ok = pair_wait_warp(acc_empty + 8 * (n & 1u), ((n >> 1) - 1u) & 1u, abort_word);
            if (!ok) break;
            tc_after();
            for (uint32_t k = 0; k < nk; ++k, ++k_all) {
                const uint32_t s = k_all % G::kStages, slot = c_all % G::kSlots, sa = tmem + G::kSf + slot * G::kSlotCols, sb = sa + 4;
                if (k % 4 == 0) {
                    ok = pair_wait_warp(sfull + 8 * slot, (c_all / G::kSlots) & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    const uint32_t at = base + G::kScales + slot * G::kSlot;
                    pair_copy_scales(sa, at, lead);
                    pair_copy_scales(sb, at + 512, lead);
                    pair_copy_scales(sb + 4, at + 1024, lead);
                }
                ok = pair_wait_warp(full + 8 * s, (k_all / G::kStages) & 1u, abort_word);
                if (!ok) break;
                tc_after();
                const uint64_t da = operand_desc(base + s * G::kStage), db = operand_desc(base + s * G::kStage + G::kA);
                const uint32_t idesc = ((k % 4) << 4) | ((G::kN >> 3) << 17) | (1u << 23) | ((256u >> 4) << 24) | ((k % 4) << 29);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) pair_mma(acc, da + 2 * i, db + 2 * i, idesc, sa, sb, (k | i) ? 1u : 0u, lead);
                pair_commit(empty + 8 * s, lead);
                if (k % 4 == 3 || k + 1u == nk) {
                    pair_commit(sempty + 8 * slot, lead);
                    ++c_all;
                }
            }
            if (!ok) break;
            pair_commit(acc_full + 8 * (n & 1u), lead);
        }
        pair_commit(done, lead);
        bar_drain(done, 0);                               // nothing is in flight when the pair ends
    } else if (warp == 1) {
    } else if (warp < 4) {
        // The scale words: byte i of a word is the scale of block k + i; row r of 128 lies at 16 (r % 32) + 4 (r / 32).  The two warps take
        // words of four blocks in turn and ask for their next ones before they wait for room (a word's products take 0.8 us, about as
        // long as its loads: one after the other they held the products up for half of the time).  Rows of x's scales that do not all begin on four
        // bytes are read byte by byte, which does hold them up: 777 x 3000 x 1744 (rows of 14) 16.1 us, with rows 16 apart 13.4.
        const bool words = (P.ldsx & 3) == 0 && (reinterpret_cast<uintptr_t>(P.sx) & 3u) == 0;
        const uint32_t per_tile = (nk + 3u) / 4u;
        uint32_t tile = pair, q = 0;                      // the tile, and which of its words
        auto step = [&](uint32_t by) {
            for (q += by; q >= per_tile && tile < tiles; q -= per_tile) tile += pairs;
        };
        uint32_t word = 0, xw[6];
        auto fetch = [&]() {
            if (tile >= tiles) return;
            const uint32_t k = 4u * q, left = min(4u, nk - k), rb = (tile % P.tiles_r) * 2u + rank, t0 = (tile / P.tiles_r) * G::kN;
            auto four = [&](const uint8_t *p, bool aligned) {
                if (aligned && left == 4) return __ldg(reinterpret_cast<const uint32_t *>(p));
                uint32_t w = 0;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (i < left) w |= uint32_t(__ldg(p + i)) << (8 * i);
                return w;
            };
            word = P.sw && rb * kBlock < P.R ? four(P.sw + int64_t(rb) * P.ldsw + k, false) : 0x7F7F7F7Fu;
#pragma unroll
            for (uint32_t j = 0; j < 6; ++j) {
                const uint32_t t = t0 + lane + 32u * j;
                xw[j] = t < P.T ? four(P.sx + int64_t(t) * P.ldsx + k, words) : 0x7F7F7F7Fu;
            }
        };
        c_all = warp - 2u;
        step(c_all);
        fetch();
        while (tile < tiles) {
            const uint32_t slot = c_all % G::kSlots, at = base + G::kScales + slot * G::kSlot;
            if (c_all >= G::kSlots) ok = bar_wait_warp(sempty + 8 * slot, (c_all / G::kSlots - 1u) & 1u, abort_word);
            if (!ok) break;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) st_smem(at + 4 * (lane + 32u * j), word);
#pragma unroll
            for (uint32_t j = 0; j < 6; ++j) st_smem(at + 512 + 512 * (j / 4) + 16 * lane + 4 * (j % 4), xw[j]);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) first_arrive(sfull + 8 * slot);
            c_all += 2u;
            step(2u);
            fetch();
        }
    } else {
        const uint32_t quarter = warp & 3u;
        for (uint32_t tile = pair; tile < tiles && ok; tile += pairs, ++n) {
            const uint32_t r = (tile % P.tiles_r) * 256u + rank * 128u + quarter * 32u + lane, t0 = (tile / P.tiles_r) * G::kN;
            ok = bar_wait_warp(acc_full + 8 * (n & 1u), (n >> 1) & 1u, abort_word);
            if (!ok) break;
            tc_after();
            const float a = P.a && r < P.R ? __ldg(P.a + r) : 1.0f;
            T *y = static_cast<T *>(P.y) + r;
#pragma unroll 1
            for (uint32_t c = 0; c < G::kN; c += 32) {
                if (t0 + c >= P.T) break;
                uint32_t v[32];
                tc_load32(tmem + (n & 1u) * G::kN + ((quarter * 32u) << 16) + c, v);
                tc_loaded32(v);
                if (r < P.R)
#pragma unroll
                    for (uint32_t i = 0; i < 32; ++i)
                        if (t0 + c + i < P.T) y[int64_t(t0 + c + i) * P.ldy] = E::of(__uint_as_float(v[i]) * a);
            }
            tc_before();
            __syncwarp();
            if (lane == 0) first_arrive(acc_empty + 8 * (n & 1u));
        }
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_matmul_status, unsigned(kStatusWait));
    cluster_sync();                                       // the other CTA's memory is read and arrived at until here
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <class E>
int launch_pair(MatmulParams P, const void *x, int64_t ldx, const void *w, int64_t ldw, uint32_t C, cudaStream_t st) {
    using G = PairShape;
    static bool configured[64] = {};
    int rc = op_configure(matmul_pair_kernel<E>, G::kSmem, configured);
    if (rc) return rc;
    CUtensorMap wm, xm;
    if ((rc = byte_map(&wm, w, C, P.R, uint64_t(ldw), 128, 128, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    if ((rc = byte_map(&xm, x, C, P.T, uint64_t(ldx), 128, G::kN / 2, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    P.tiles_r = (P.R + 255u) / 256u;
    const uint64_t tiles = uint64_t(P.tiles_r) * ((P.T + G::kN - 1u) / G::kN);
    if (tiles > 0x7FFFFFFFu || tiles * P.blocks > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    const uint32_t pairs = uint32_t(op_sms()) / 2u, grid = 2u * uint32_t(tiles < pairs ? tiles : pairs);
    return op_launch(matmul_pair_kernel<E>, grid, 256, G::kSmem, 1, st, P, wm, xm) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

template <class E>
int launch_matmul(const MatmulParams &P, const void *x, int64_t ldx, const void *w, int64_t ldw, uint32_t C, cudaStream_t st) {
    if (P.T <= 16) return launch_split<16, E>(P, x, ldx, w, ldw, C, st);
    if (P.T <= 32) return launch_split<32, E>(P, x, ldx, w, ldw, C, st);
    // (up to 128 tokens as two tiles of 64 where three CTAs can share each: 4096^2 8.8 us instead of 11.1, 512^2 6.3 / 8.8; without that 8192^2 21.1 / 20.0)
    if (P.T <= 64 || (P.T <= 128 && 6ull * P.tiles_r <= 2ull * uint64_t(op_sms()))) return launch_split<64, E>(P, x, ldx, w, ldw, C, st);
    // Estimates in units of 10 ns, fitted to 129 - 1024 tokens x 1024^2 .. 8192^2, 3000 x 1744 and 2048 x 17408: pairs take a round of all SMs
    // after another, clusters share out blocks of columns.  us, pairs / clusters: 256 tokens x 1024^2 9.3 / 7.4, x 4096^2 15.3 / 13.4, x 8192^2
    // 26.3 / 33.8, x 2048 x 17408 41.2 / 20.8, 1024 tokens 9.6 / 10.8, 24.7 / 23.8, 68 / 91, 42.7 / 60.4.
    const int sms = op_sms();
    if (sms <= 1) return EP_ERR_CUDA;
    const uint64_t pairs = uint64_t(sms) / 2u, pair_tiles = uint64_t((P.R + 255u) / 256u) * ((P.T + PairShape::kN - 1u) / PairShape::kN),
                   split_tiles = uint64_t(P.tiles_r) * ((P.T + 127u) / 128u);
    const uint64_t by_pairs = 470u + (pair_tiles + pairs - 1u) / pairs * (27ull * P.blocks + 250u), by_clusters = 800u + 40ull * split_tiles * P.blocks / uint64_t(sms);
    if (by_pairs < by_clusters) return launch_pair<E>(P, x, ldx, w, ldw, C, st);
    return launch_split<128, E>(P, x, ldx, w, ldw, C, st);
}

const bool registered = ep::add_status_word([] { return op_status(g_matmul_status); });

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

}  // namespace

extern "C" int ep_quantize_blocks(const ep_quantize_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_quantize_job &j = *job;
    if (j.T == 0) return EP_OK;
    if (!j.d_x || !j.d_q || !j.d_scales || j.C == 0 || j.C > 0x7FFFFF00u || (j.block_rows != 1 && j.block_rows != kBlock)) return EP_ERR_BAD_ARG;
    const uint32_t size = j.x_dtype == EP_FP32 ? 4 : j.x_dtype == EP_BF16 || j.x_dtype == EP_FP16 ? 2 : 0;
    if (!size || !aligned(j.d_x, size)) return EP_ERR_BAD_ARG;
    QuantParams P;
    std::memset(&P, 0, sizeof(P));
    P.blocks = (j.C + kBlock - 1u) / kBlock;
    if (j.ldx < int64_t(j.C) || j.ldq < int64_t(j.C) || j.lds < int64_t(P.blocks)) return EP_ERR_BAD_ARG;
    P.x = j.d_x;
    P.q = static_cast<uint8_t *>(j.d_q);
    P.s = static_cast<uint8_t *>(j.d_scales);
    P.ldx = j.ldx;
    P.ldq = j.ldq;
    P.lds = j.lds;
    P.T = j.T;
    P.C = j.C;
    P.vec = aligned(j.d_x, 16) && j.ldx * size % 16 == 0 && aligned(j.d_q, 16) && j.ldq % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (j.x_dtype == EP_BF16) return launch_quantize<Bf16>(P, j.block_rows, st);
    if (j.x_dtype == EP_FP16) return launch_quantize<Fp16>(P, j.block_rows, st);
    return launch_quantize<Fp32>(P, j.block_rows, st);
}

extern "C" int ep_fp8_matmul(const ep_matmul_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_matmul_job &j = *job;
    if (j.T == 0) return EP_OK;
    if (!j.d_x || !j.d_x_scales || !j.d_w || !j.d_y || j.R == 0 || j.C == 0 || j.C > 0x7FFFFF00u || j.R > 0x7FFFFF00u || j.T > 0x7FFFFF00u) return EP_ERR_BAD_ARG;
    const uint32_t size = j.out_dtype == EP_FP32 ? 4 : j.out_dtype == EP_BF16 || j.out_dtype == EP_FP16 ? 2 : 0;
    const uint32_t blocks = (j.C + kBlock - 1u) / kBlock;
    if (!size || !aligned(j.d_y, size) || (j.d_row_scales && !aligned(j.d_row_scales, 4)) || j.ldx < int64_t(j.C) || j.ldw < int64_t(j.C) ||
        j.ldx_scales < int64_t(blocks) || (j.d_w_scales && j.ldw_scales < int64_t(blocks)) || j.ldy < int64_t(j.R))
        return EP_ERR_BAD_ARG;
    // the copy engine's rows begin on 16 bytes
    if (j.C % 16 || j.ldx % 16 || j.ldw % 16 || !aligned(j.d_x, 16) || !aligned(j.d_w, 16) || j.ldx >= (int64_t(1) << 40) || j.ldw >= (int64_t(1) << 40))
        return EP_ERR_UNSUPPORTED;
    MatmulParams P;
    std::memset(&P, 0, sizeof(P));
    P.sx = static_cast<const uint8_t *>(j.d_x_scales);
    P.sw = static_cast<const uint8_t *>(j.d_w_scales);
    P.a = j.d_row_scales;
    P.y = j.d_y;
    P.ldsx = j.ldx_scales;
    P.ldsw = j.ldw_scales;
    P.ldy = j.ldy;
    P.T = j.T;
    P.R = j.R;
    P.blocks = blocks;
    P.tiles_r = (j.R + kBlock - 1u) / kBlock;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (j.out_dtype == EP_BF16) return launch_matmul<Bf16>(P, j.d_x, j.ldx, j.d_w, j.ldw, j.C, st);
    if (j.out_dtype == EP_FP16) return launch_matmul<Fp16>(P, j.d_x, j.ldx, j.d_w, j.ldw, j.C, st);
    return launch_matmul<Fp32>(P, j.d_x, j.ldx, j.d_w, j.ldw, j.C, st);
}
