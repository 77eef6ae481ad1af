// Rounding to INT8 row by row, and the matrix product of operands held that way.
#include "op_rows.hpp"

using namespace ep;

namespace {

constexpr uint32_t kBlock = 128;                 // columns of a stage: bytes of a swizzled row
__device__ unsigned int g_int8_status = 0;

// ======================================================================================================================
// Rounding: m = max(max |x|, 2^-119), s = m / 127, q = round(x * (127 / m)).  One division a row; q is a whole number's distance of half from
// x / s but for the last bits of 127 / m, which no INT8 grid notices.
// Bound by memory: rows of up to 32768 values wait in registers for their maximum, longer ones are read twice.
// ======================================================================================================================
struct RowsParams {
    const uint8_t *x;
    uint8_t *q;
    float *s;
    int64_t ldx, ldq;             // bytes
    uint32_t T, C;
    uint32_t warps, rows;         // warps of a row, rows of a CTA
    int32_t half;
    uint32_t x_vec, q_vec;
};

template <uint32_t BITS>
__device__ __forceinline__ uint32_t largest_bits(const Eight<BITS> &e, bool half) {     // as a float's
    uint32_t a = 0;
    if constexpr (BITS == 32) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) a = max(a, e.w[i] & 0x7FFFFFFFu);
        return a;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) a = __vmaxu2(a, e.w[i] & 0x7FFF7FFFu);
        a = max(a & 0xFFFFu, a >> 16);
        return __float_as_uint(half ? Fp16::lo(a) : Bf16::lo(a));
    }
}
template <uint32_t BITS>
__device__ __forceinline__ void store_int8(const Eight<BITS> &e, bool half, const Int8Scale &s, uint8_t *row, uint32_t c, uint32_t n, bool vec) {
    Pair v[4];
    to_pairs<BITS>(e, half, v);
    uint32_t lo, hi;
    to_int8(v, s.inverse, lo, hi);
    if (s.s != s.s) lo = hi = 0;
    store_bytes(row, c, n, vec, lo, hi);
}

template <uint32_t BITS, uint32_t N>
__global__ void __launch_bounds__(512) quantize_rows_kernel(const __grid_constant__ RowsParams P) {
    __shared__ uint32_t room[64];
    op_wait_for_stream();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, of = warp / P.warps;
    const uint32_t row = blockIdx.x * P.rows + of, l = (warp - of * P.warps) * 32u + lane;
    RowGroup group{room, P.warps, of * P.warps, 1u + of, 0};
    const uint8_t *x = P.x + int64_t(row) * P.ldx;
    Eight<BITS> e[N];
    uint32_t top = 0;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t c = (i * P.warps * 32u + l) * 8u;
        load_eight<BITS>(x, c, row < P.T ? inside(c, P.C) : 0u, P.x_vec, e[i]);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) top = max(top, largest_bits<BITS>(e[i], P.half));
    const Int8Scale s = int8_scale(group.largest(top));
    if (row >= P.T) return;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t c = (i * P.warps * 32u + l) * 8u;
        store_int8<BITS>(e[i], P.half, s, P.q + int64_t(row) * P.ldq, c, inside(c, P.C), P.q_vec);
    }
    if (l == 0) P.s[row] = s.s;
}
template <uint32_t BITS>
__global__ void __launch_bounds__(512) quantize_long_rows_kernel(const __grid_constant__ RowsParams P) {
    __shared__ uint32_t room[64];
    op_wait_for_stream();
    RowGroup group{room, P.warps, 0, 1, 0};
    const uint8_t *x = P.x + int64_t(blockIdx.x) * P.ldx;
    uint32_t top = 0;
    Eight<BITS> e;
#pragma unroll 4
    for (uint32_t c = threadIdx.x * 8u; c < P.C; c += blockDim.x * 8u) {
        load_eight<BITS, true>(x, c, inside(c, P.C), P.x_vec, e);
        top = max(top, largest_bits<BITS>(e, P.half));
    }
    const Int8Scale s = int8_scale(group.largest(top));
#pragma unroll 4
    for (uint32_t c = threadIdx.x * 8u; c < P.C; c += blockDim.x * 8u) {
        load_eight<BITS>(x, c, inside(c, P.C), P.x_vec, e);
        store_int8<BITS>(e, P.half, s, P.q + int64_t(blockIdx.x) * P.ldq, c, inside(c, P.C), P.q_vec);
    }
    if (threadIdx.x == 0) P.s[blockIdx.x] = s.s;
}

template <uint32_t BITS>
int launch_rows(RowsParams P, cudaStream_t st) {
    const uint32_t pieces = (P.C + 7u) / 8u;
    const uint32_t each = pieces <= 512 ? 1u : pieces <= 1024 ? 2u : pieces <= 2048 ? 4u : 8u;
    if (pieces > 4096) {
        P.warps = 16, P.rows = 1;
        return op_launch(quantize_long_rows_kernel<BITS>, P.T, 512, 0, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
    }
    P.warps = (pieces + 32u * each - 1u) / (32u * each);
    P.rows = P.warps >= 4 ? 1u : 4u / P.warps;
    const uint32_t threads = P.warps * P.rows * 32u, grid = uint32_t((uint64_t(P.T) + P.rows - 1u) / P.rows);
    const cudaError_t e = each == 1 ? op_launch(quantize_rows_kernel<BITS, 1>, grid, threads, 0, 1, st, P)
                        : each == 2 ? op_launch(quantize_rows_kernel<BITS, 2>, grid, threads, 0, 1, st, P)
                        : each == 4 ? op_launch(quantize_rows_kernel<BITS, 4>, grid, threads, 0, 1, st, P)
                                    : op_launch(quantize_rows_kernel<BITS, 8>, grid, threads, 0, 1, st, P);
    return e == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// ======================================================================================================================
// y[t, r] = a[r] (s[t] sum_k xq[t, k] wq[r, k]) + bias[r]
//
// On the tensor cores as D = A B^T with A = rows of the weight (a single token still fills the instruction's 128 lanes) and B =
// tokens: tcgen05.mma kind::i8, products of whole numbers summed in 32 bits, exactly, so that sums may be split in any way and come out the same.
// ======================================================================================================================
struct ProductParams {
    const float *s, *a, *bias;    // a, bias may be null
    void *y;
    int64_t ldy;
    uint32_t T, R, blocks;        // blocks = ceil(C / 128)
    uint32_t rows, strips;        // rows of the weight to a strip, strips: a grid walks them first
    uint32_t split;               // CTAs (one cluster) that share a strip's columns
    uint32_t stages, stage;       // in shared memory; bytes of one
};

// the epilogue, the same in every kernel so that results do not depend on which one is taken
__device__ __forceinline__ float scaled(uint32_t sum, float s, float a, float bias) { return fmaf(a, s * float(int32_t(sum)), bias); }

// S32 sums of S8 x S8, both K-major, M = m, N = n
__host__ __device__ constexpr uint32_t i8_idesc(uint32_t m, uint32_t n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((m >> 4) << 24); }
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}
__device__ __forceinline__ void pair_mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}

// ---- few tokens: a strip of rows per CTA ------------------------------------------------------------------------------------
// The weight's bytes bound it, so every SM has to have an equal share of them and some tens of KB in flight.  A CTA takes a strip of up to 128 rows, however
// many make the shares equal (the instruction's other lanes are computed from whatever follows in shared memory and never read).  Where a
// strip would be so low that the tokens' bytes, which every CTA reads, outgrow the weight's, a cluster of CTAs shares the
// columns of a higher strip; at the end they lay their sums down in shared memory and each adds up its share of the tokens over the cluster.
template <uint32_t BN>
struct StripShape {
    static constexpr uint32_t kB = BN * 128, kMaxStages = 16, kRoom = 96 * 1024;      // bytes of stages: two CTAs fit an SM
    static constexpr uint32_t kTail = 128 * 128;                                       // what the last stage's instructions may read beyond it
    static constexpr uint32_t kBars = kRoom + kTail - 8 * 128, kScales = kBars + 16 * kMaxStages + 32, kSmem = kScales + 4 * BN + 1024;
    static_assert(2 * (kSmem + 1024) <= 228 * 1024);
    static constexpr uint32_t kCols = BN < 32 ? 32 : BN;
};

template <uint32_t BN, class E>
__global__ void __launch_bounds__(128) product_strip_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ CUtensorMap w_map,
                                                            const __grid_constant__ CUtensorMap x_map) {
    using G = StripShape<BN>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t full = base + G::kBars, empty = full + 8 * G::kMaxStages, done = empty + 8 * G::kMaxStages, slot_addr = done + 8, abort_word = slot_addr + 4,
                   scales = base + G::kScales;
    if (tid == 0) {
        for (uint32_t i = 0; i < P.stages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
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
    const uint32_t tmem = ld_smem(slot_addr);
    const uint32_t tile = blockIdx.x / P.split, rank = blockIdx.x % P.split;
    const uint32_t strip = tile % P.strips, t0 = (tile / P.strips) * BN;
    // strips of equal height, but for one row
    const uint32_t r0 = uint32_t(uint64_t(P.R) * strip / P.strips), r1 = uint32_t(uint64_t(P.R) * (strip + 1) / P.strips);
    const uint32_t kb0 = P.blocks * rank / P.split, kb1 = P.blocks * (rank + 1) / P.split, nk = kb1 - kb0;
    const uint32_t r = r0 + tid;
    float a = 1.0f, bias = 0.0f;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t k = 0, s = 0, phase = 1;
            for (; k < nk; ++k) {
                const uint32_t at = base + s * P.stage;
                if (k >= P.stages && !bar_wait(empty + 8 * s, phase, abort_word)) break;
                bar_expect(full + 8 * s, P.rows * 128 + G::kB);
                tma_load_2d(at + G::kB, &w_map, int32_t((kb0 + k) * 128u), int32_t(r0), full + 8 * s);
                tma_load_2d(at, &x_map, int32_t((kb0 + k) * 128u), int32_t(t0), full + 8 * s);
                if (++s == P.stages) s = 0, phase ^= 1u;
            }
            if (ld_smem(abort_word))                     // nothing may land after the CTA's end
                for (uint32_t j = k > P.stages ? k - P.stages : 0; j < k; ++j) bar_drain(full + 8 * (j % P.stages), (j / P.stages) & 1u);
        }
    } else if (warp == 1) {
        const uint32_t lead = elected();
        uint32_t s = 0, phase = 0;
        for (uint32_t k = 0; k < nk; ++k) {
            if (!bar_wait_warp(full + 8 * s, phase, abort_word)) break;
            tc_after();
            const uint32_t at = base + s * P.stage;
            const uint64_t da = operand_desc(at + G::kB), db = operand_desc(at);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) mma_i8(tmem, da + 2 * i, db + 2 * i, i8_idesc(128, BN), (k | i) ? 1u : 0u, lead);
            tc_commit(empty + 8 * s, lead);
            if (++s == P.stages) s = 0, phase ^= 1u;
        }
        tc_commit(done, lead);
    } else {
        for (uint32_t t = tid - 64u; t < BN; t += 64) st_smem(scales + 4 * t, __float_as_uint(t0 + t < P.T ? __ldg(P.s + t0 + t) : 0.0f));
    }
    if (P.split == 1 && r < r1) {
        if (P.a) a = __ldg(P.a + r);
        if (P.bias) bias = __ldg(P.bias + r);
    }
    __syncthreads();
    bar_wait(done, 0, abort_word);
    if (ld_smem(abort_word)) bar_drain(done, 0);         // instructions in flight still read the stages
    tc_after();

    // lane = row of the weight, register = token
    if (P.split == 1) {
        T *y = static_cast<T *>(P.y) + r;
#pragma unroll
        for (uint32_t c = 0; c < BN; c += 16) {
            if (t0 + c >= P.T) break;
            uint32_t v[16];
            tc_load16(tmem + ((warp * 32u) << 16) + c, v);
            tc_loaded16(v);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (r < r1 && t0 + c + i < P.T) y[int64_t(t0 + c + i) * P.ldy] = E::of(scaled(v[i], __uint_as_float(ld_smem(scales + 4 * (c + i))), a, bias));
        }
    } else {
#pragma unroll
        for (uint32_t c = 0; c < BN; c += 16) {
            uint32_t v[16];
            tc_load16(tmem + ((warp * 32u) << 16) + c, v);
            tc_loaded16(v);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) st_smem(base + ((c + i) * 128u + tid) * 4u, v[i]);
        }
        cluster_sync();
        // this CTA's tokens, one to a warp, four rows to a lane; all CTAs' parts asked for at once
        const uint32_t c0 = BN * rank / P.split, c1 = BN * (rank + 1) / P.split, r4 = r0 + 4u * lane;
        uint32_t peer[8];
        float a4[4], b4[4];
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer[p]) : "r"(base), "r"(min(p, P.split - 1u)));
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            a4[j] = P.a && r4 + j < r1 ? __ldg(P.a + r4 + j) : 1.0f;
            b4[j] = P.bias && r4 + j < r1 ? __ldg(P.bias + r4 + j) : 0.0f;
        }
#pragma unroll 2
        for (uint32_t c = c0 + warp; c < c1; c += 4) {
            if (t0 + c >= P.T) break;
            int4 v[8];
#pragma unroll
            for (uint32_t p = 0; p < 8; ++p)
                if (p < P.split)
                    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v[p].x), "=r"(v[p].y), "=r"(v[p].z), "=r"(v[p].w) : "r"(peer[p] + (c * 128u + 4u * lane) * 4u) : "memory");
            int32_t sum[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (uint32_t p = 1; p < 8; ++p)
                if (p < P.split) sum[0] += v[p].x, sum[1] += v[p].y, sum[2] += v[p].z, sum[3] += v[p].w;
            const float s = __uint_as_float(ld_smem(scales + 4 * c));
            T *dst = static_cast<T *>(P.y) + int64_t(t0 + c) * P.ldy + r4;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (r4 + j < r1) dst[j] = E::of(scaled(uint32_t(sum[j]), s, a4[j], b4[j]));
        }
        cluster_sync();
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_int8_status, unsigned(kStatusWait));
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kCols) : "memory");
}

struct Operands {
    const void *x, *w;
    int64_t ldx, ldw;
    uint32_t C;
};

template <uint32_t BN, class E>
int launch_strip(ProductParams P, const Operands &o, uint32_t split, cudaStream_t st) {
    using G = StripShape<BN>;
    static bool configured[64] = {};
    int rc = op_configure(product_strip_kernel<BN, E>, G::kSmem, configured);
    if (rc) return rc;
    const uint32_t sms = uint32_t(op_sms());
    if (!sms) return EP_ERR_CUDA;
    const uint64_t tiles_t = (P.T + BN - 1u) / BN;
    P.split = split;
    // as many strips as make one CTA on each SM, or a whole number of them where strips of 128 rows are more
    const uint64_t least = (uint64_t(P.R) + 127u) / 128u, round = sms / split / tiles_t;
    uint64_t strips = round ? (least + round - 1u) / round * round : least;
    if (strips > P.R) strips = P.R;
    P.strips = uint32_t(strips);
    P.rows = (P.R + P.strips - 1u) / P.strips;
    if (P.rows > 128) return EP_ERR_UNSUPPORTED;
    P.stage = (P.rows + 7u) / 8u * 1024u + G::kB;
    P.stages = G::kRoom / P.stage;
    if (P.stages > G::kMaxStages) P.stages = G::kMaxStages;
    CUtensorMap wm, xm;
    if ((rc = byte_map(&wm, o.w, o.C, P.R, uint64_t(o.ldw), 128, P.rows, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    if ((rc = byte_map(&xm, o.x, o.C, P.T, uint64_t(o.ldx), 128, BN, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    const uint64_t grid = uint64_t(P.strips) * tiles_t * split;
    if (grid > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    return op_launch(product_strip_kernel<BN, E>, uint32_t(grid), 128, G::kSmem, split, st, P, wm, xm) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// ---- many tokens: a pair of CTAs per tile -----------------------------------------------------------------------------------
// Two CTAs share tiles of 256 rows of the weight by N tokens (tcgen05 cta_group::2): each has half of the weight's rows and half of the tokens
// in its shared memory, and keeps the sums of its 128 rows with all tokens in its tensor memory, twice, so that a tile is read out while the next one
// is summed.
//   warp 0        brings the operands in
//   warp 1        of the first CTA issues the products
//   warps 4 - 7   sums to y
template <uint32_t N>
struct PairShape {
    static constexpr uint32_t kA = kBlock * 128, kB = N / 2 * 128, kStage = kA + kB, kStages = N == 256 ? 7 : 9;
    static constexpr uint32_t kBars = kStages * kStage, kSmem = kBars + 512 + 1024, kCols = 2 * N;
    static_assert(kSmem <= 232448 && kCols <= 512);
};

template <uint32_t N, class E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(256, 1)
    product_pair_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map) {
    using G = PairShape<N>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t rank = blockIdx.x & 1u, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t full = base + G::kBars, empty = full + 8 * G::kStages, acc_full = empty + 8 * G::kStages, acc_empty = acc_full + 16, done = acc_empty + 16,
                   slot_addr = done + 8, abort_word = slot_addr + 4;
    if (tid == 0) {
        for (uint32_t i = 0; i < G::kStages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (uint32_t i = 0; i < 2; ++i) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, 8);
        bar_init(done, 1);
        st_smem(abort_word, 0);
        bar_init_done();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(G::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_sync();                                       // the other CTA's barriers are there
    tc_after();
    op_wait_for_stream();
    const uint32_t tmem = ld_smem(slot_addr);
    const uint32_t tiles = P.strips * ((P.T + N - 1u) / N), nk = P.blocks;
    uint32_t k_all = 0, n = 0;                            // blocks and tiles so far
    bool ok = true;

    if (warp == 0) {
        for (uint32_t tile = pair; tile < tiles && ok; tile += pairs) {
            const uint32_t r0 = (tile % P.strips) * 256u + rank * 128u, t0 = (tile / P.strips) * N + rank * (N / 2);
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
            const uint32_t acc = tmem + (n & 1u) * N;
            if (n > 1u) ok = pair_wait_warp(acc_empty + 8 * (n & 1u), ((n >> 1) - 1u) & 1u, abort_word);
            if (!ok) break;
            tc_after();
            for (uint32_t k = 0; k < nk; ++k, ++k_all) {
                const uint32_t s = k_all % G::kStages;
                ok = pair_wait_warp(full + 8 * s, (k_all / G::kStages) & 1u, abort_word);
                if (!ok) break;
                tc_after();
                const uint64_t da = operand_desc(base + s * G::kStage), db = operand_desc(base + s * G::kStage + G::kA);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) pair_mma_i8(acc, da + 2 * i, db + 2 * i, i8_idesc(256, N), (k | i) ? 1u : 0u, lead);
                pair_commit(empty + 8 * s, lead);
            }
            if (!ok) break;
            pair_commit(acc_full + 8 * (n & 1u), lead);
        }
        pair_commit(done, lead);
        bar_drain(done, 0);                               // nothing is in flight when the pair ends
    } else if (warp >= 4) {
        const uint32_t quarter = warp & 3u;
        for (uint32_t tile = pair; tile < tiles && ok; tile += pairs, ++n) {
            const uint32_t r = (tile % P.strips) * 256u + rank * 128u + quarter * 32u + lane, t0 = (tile / P.strips) * N;
            const float a = P.a && r < P.R ? __ldg(P.a + r) : 1.0f, bias = P.bias && r < P.R ? __ldg(P.bias + r) : 0.0f;
            float s[N / 32];                              // of token t0 + 32 i + lane
#pragma unroll
            for (uint32_t i = 0; i < N / 32; ++i) s[i] = t0 + 32 * i + lane < P.T ? __ldg(P.s + t0 + 32 * i + lane) : 0.0f;
            ok = bar_wait_warp(acc_full + 8 * (n & 1u), (n >> 1) & 1u, abort_word);
            if (!ok) break;
            tc_after();
            T *y = static_cast<T *>(P.y) + r;
#pragma unroll
            for (uint32_t c = 0; c < N; c += 32) {
                if (t0 + c >= P.T) break;
                uint32_t v[32];
                tc_load32(tmem + (n & 1u) * N + ((quarter * 32u) << 16) + c, v);
                tc_loaded32(v);
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i) {
                    const float f = scaled(v[i], __shfl_sync(0xFFFFFFFFu, s[c / 32], i), a, bias);
                    if (r < P.R && t0 + c + i < P.T) y[int64_t(t0 + c + i) * P.ldy] = E::of(f);
                }
            }
            tc_before();
            __syncwarp();
            if (lane == 0) first_arrive(acc_empty + 8 * (n & 1u));
        }
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_int8_status, unsigned(kStatusWait));
    cluster_sync();                                       // the other CTA's memory is read and arrived at until here
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kCols) : "memory");
    }
}

template <uint32_t N, class E>
int launch_pair(ProductParams P, const Operands &o, cudaStream_t st) {
    using G = PairShape<N>;
    static bool configured[64] = {};
    int rc = op_configure(product_pair_kernel<N, E>, G::kSmem, configured);
    if (rc) return rc;
    CUtensorMap wm, xm;
    if ((rc = byte_map(&wm, o.w, o.C, P.R, uint64_t(o.ldw), 128, 128, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    if ((rc = byte_map(&xm, o.x, o.C, P.T, uint64_t(o.ldx), 128, N / 2, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
    P.strips = (P.R + 255u) / 256u;
    const uint64_t tiles = uint64_t(P.strips) * ((P.T + N - 1u) / N);
    if (tiles > 0x7FFFFFFFu || tiles * P.blocks > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    const uint32_t pairs = uint32_t(op_sms()) / 2u, grid = 2u * uint32_t(tiles < pairs ? tiles : pairs);
    return op_launch(product_pair_kernel<N, E>, grid, 256, G::kSmem, 1, st, P, wm, xm) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

template <class E>
int launch_product(const ProductParams &P, const Operands &o, cudaStream_t st) {
    if (P.T <= 16) return launch_strip<16, E>(P, o, 1, st);
    if (P.T <= 32) return launch_strip<32, E>(P, o, 1, st);
    if (P.T <= 64) return launch_strip<64, E>(P, o, 1, st);
    if (P.T <= 128) return launch_strip<128, E>(P, o, 1, st);
    return launch_pair<256, E>(P, o, st);
}

const bool registered = ep::add_status_word([] { return op_status(g_int8_status); });

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

}  // namespace

extern "C" int ep_quantize_rows(const ep_quantize_rows_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_quantize_rows_job &j = *job;
    if (j.T == 0) return EP_OK;
    const uint32_t size = j.x_dtype == EP_FP32 ? 4 : j.x_dtype == EP_BF16 || j.x_dtype == EP_FP16 ? 2 : 0;
    if (!j.d_x || !j.d_q || !j.d_scales || j.C == 0 || j.C > 0x7FFFFF00u || j.T > 0x7FFFFF00u || !size || !aligned(j.d_x, size) || !aligned(j.d_scales, 4) ||
        j.ldx < int64_t(j.C) || j.ldq < int64_t(j.C) || j.ldx >= (int64_t(1) << 40) || j.ldq >= (int64_t(1) << 40))
        return EP_ERR_BAD_ARG;
    RowsParams P;
    std::memset(&P, 0, sizeof(P));
    P.x = static_cast<const uint8_t *>(j.d_x);
    P.q = static_cast<uint8_t *>(j.d_q);
    P.s = j.d_scales;
    P.ldx = j.ldx * size;
    P.ldq = j.ldq;
    P.T = j.T;
    P.C = j.C;
    P.half = j.x_dtype == EP_FP16;
    P.x_vec = aligned(j.d_x, 16) && P.ldx % 16 == 0;
    P.q_vec = aligned(j.d_q, 8) && j.ldq % 8 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return size == 4 ? launch_rows<32>(P, st) : launch_rows<16>(P, st);
}

extern "C" int ep_int8_matmul(const ep_int8_matmul_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_int8_matmul_job &j = *job;
    if (j.T == 0) return EP_OK;
    const uint32_t size = j.out_dtype == EP_FP32 ? 4 : j.out_dtype == EP_BF16 || j.out_dtype == EP_FP16 ? 2 : 0;
    if (!j.d_x || !j.d_x_scales || !j.d_w || !j.d_y || j.R == 0 || j.C == 0 || j.R > 0x7FFFFF00u || j.T > 0x7FFFFF00u || !size || !aligned(j.d_y, size) ||
        !aligned(j.d_x_scales, 4) || (j.d_row_scales && !aligned(j.d_row_scales, 4)) || (j.d_bias && !aligned(j.d_bias, 4)) || j.ldx < int64_t(j.C) ||
        j.ldw < int64_t(j.C) || j.ldy < int64_t(j.R))
        return EP_ERR_BAD_ARG;
    // the copy engine's rows begin on 16 bytes; sums of 128 * 128 * C stay below 2^31
    if (j.C % 16 || j.C >= (1u << 17) || j.ldx % 16 || j.ldw % 16 || !aligned(j.d_x, 16) || !aligned(j.d_w, 16) || j.ldx >= (int64_t(1) << 40) || j.ldw >= (int64_t(1) << 40))
        return EP_ERR_UNSUPPORTED;
    ProductParams P;
    std::memset(&P, 0, sizeof(P));
    P.s = j.d_x_scales;
    P.a = j.d_row_scales;
    P.bias = j.d_bias;
    P.y = j.d_y;
    P.ldy = j.ldy;
    P.T = j.T;
    P.R = j.R;
    P.blocks = (j.C + kBlock - 1u) / kBlock;
    const Operands o{j.d_x, j.d_w, j.ldx, j.ldw, j.C};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (j.out_dtype == EP_BF16) return launch_product<Bf16>(P, o, st);
    if (j.out_dtype == EP_FP16) return launch_product<Fp16>(P, o, st);
    return launch_product<Fp32>(P, o, st);
}
