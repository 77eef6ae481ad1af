// Rounding to INT8 row by row, and the matrix product of operands held that way.
#include "op_rows.hpp"

using namespace ep;

namespace {

constexpr uint32_t kBlock = 128;                 // columns of a stage: bytes of a swizzled row
__device__ unsigned int g_int8_status = 0;

// ======================================================================================================================
// Rounding: m = max(max |x|, 2^-119), s = m / 127, q = round(x * (127 / m)).  One division a row; q is a whole number's distance of half from
// x / s but for the last bits of 127 / m, which no INT8 grid notices.
// Bound by memory: rows of up to 32768 values wait in registers for their maximum (5120 x 17408 FP32 in 69.8 us, 6.4 TB/s), longer ones are read twice.
// ======================================================================================================================
struct RowsParams {
    const uint8_t *x;
    uint8_t *q;
    float *s;
    int64_t ldx, ldq;             // bytes
    uint32_t T, C;
    uint32_t warps, rows;         // warps of a row, rows of a CTA
    uint32_t lanes;               // of a row that takes less than a warp (32: whole warps)
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
    const uint32_t of = P.lanes < 32 ? threadIdx.x / P.lanes : (threadIdx.x >> 5) / P.warps;
    const uint32_t row = blockIdx.x * P.rows + of, l = threadIdx.x - of * (P.lanes < 32 ? P.lanes : P.warps * 32u);
    RowGroup group{room, P.warps, of * P.warps, 1u + of, 0, P.lanes};
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
    // Few rows are spread over many lanes; of many, a row of up to 2048 values is a warp's and one of 4096 two warps' (spread and not, us: 160000 x 128 BF16 87 / 43,
    // 40000 x 1024 86 / 36, 8192 x 3840 32 / 25, 8192 x 5120 33 / 42).
    const bool many = P.T >= 8u * uint32_t(op_sms());
    const uint32_t each = many && pieces <= 512 ? (pieces <= 32 ? 1u : pieces <= 64 ? 2u : pieces <= 128 ? 4u : 8u) : pieces <= 512 ? 1u : pieces <= 1024 ? 2u : pieces <= 2048 ? 4u : 8u;
    P.lanes = 32;
    while (P.lanes / 2 >= pieces) P.lanes /= 2;
    if (pieces > 4096) {
        P.warps = 16, P.rows = 1;
        return op_launch(quantize_long_rows_kernel<BITS>, P.T, 512, 0, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
    }
    P.warps = (pieces + 32u * each - 1u) / (32u * each);
    P.rows = P.warps >= 4 ? 1u : 4u / P.warps * (32u / P.lanes);
    const uint32_t threads = P.warps * P.rows * P.lanes, grid = uint32_t((uint64_t(P.T) + P.rows - 1u) / P.rows);
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
    uint32_t strips;              // of rows of the weight: a grid walks them first
    uint32_t split;               // CTAs (one cluster) that share a strip's columns
    uint32_t stages, stage;       // in shared memory; bytes of one
    uint32_t whole, chunk;        // whole blocks of 128 columns; how many of them a stage holds
    uint32_t m;                   // rows of the instruction: 64 or 128
    uint32_t sums;                // where a cluster's sums go, behind the stages
    uint32_t x_block, w_block;    // bytes of a block: rows in whole eights
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
// columns of a higher strip; at the end they send one another their sums, and each adds up its share of the tokens.
//   warp 0       brings chunks of up to four blocks of 128 columns in, with one request for each operand (the blocks are a tensor's third dimension)
//   warp 1       issues the products; M = 64 for strips of up to 64 rows: the instruction reads its 128 rows at 64 bytes a cycle, whether they are real or not
//   warps 2, 3   the tokens' scales; all four warps read the sums out
// 10240 x 3840 by 1 token 9.4 us (5.5 TB/s while it runs; 2.5 us are the change of kernels and the first bytes), 5120 x 17408 by 1 token 17.8, by 48 19.7 (each
// SM's way from L2, which brings all tokens), 1024 x 8192 by 32 in clusters of eight 5.3.
template <uint32_t BN>
struct StripShape {
    static constexpr uint32_t kMaxStages = 32, kTail = 128 * 128;       // kTail: what the last stage's instructions may read beyond it
    static constexpr uint32_t kBars = 0, kScales = 16 * kMaxStages + 16, kStages = 2048;
    static constexpr uint32_t kSmem(uint32_t stages, uint32_t stage) { return kStages + stages * stage + kTail + 1024; }
    static constexpr uint32_t kMost = 226 * 1024;
    static constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    static_assert(kScales + 4 * BN <= kStages && BN <= 128);
};

// Sixteen tokens' sums from tensor memory to y, a row of the weight to each lane; the first n tokens are there.  Token i's scale lies at scales + 4 i.
template <class E>
__device__ __forceinline__ void put_sixteen(uint32_t tmem, uint32_t scales, typename E::T *y, int64_t ldy, uint32_t n, float a, float bias) {
    uint32_t v[16];
    uint4 f[4];
    tc_load16(tmem, v);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) f[i] = ld_smem16(scales + 16 * i);
    tc_loaded16(v);
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i, y += ldy) {
        const uint4 g = f[i / 4];
        const uint32_t s = i % 4 == 0 ? g.x : i % 4 == 1 ? g.y : i % 4 == 2 ? g.z : g.w;
        if (i < n) *y = E::of(scaled(v[i], __uint_as_float(s), a, bias));
    }
}

template <uint32_t BN, class E>
__global__ void __launch_bounds__(128)
    product_strip_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
                         const __grid_constant__ CUtensorMap w_tail, const __grid_constant__ CUtensorMap x_tail) {
    using G = StripShape<BN>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t full = base + G::kBars, empty = full + 8 * G::kMaxStages, done = empty + 8 * G::kMaxStages, slot_addr = done + 8, abort_word = slot_addr + 4,
                   scales = base + G::kScales, ring = base + G::kStages;
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
    if (P.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");        // (this CTA has begun)
    const uint32_t tile = blockIdx.x / P.split, rank = blockIdx.x % P.split;
    const uint32_t strip = tile % P.strips, t0 = (tile / P.strips) * BN;
    // strips of equal height, but for one row
    const uint32_t r0 = uint32_t(uint64_t(P.R) * strip / P.strips), r1 = uint32_t(uint64_t(P.R) * (strip + 1) / P.strips);
    // chunks of whole blocks, and what is left of the columns as one of its own
    const uint32_t chunks = (P.whole + P.chunk - 1u) / P.chunk + (P.blocks - P.whole);
    const uint32_t k0 = chunks * rank / P.split, nk = chunks * (rank + 1) / P.split - k0;
    op_wait_for_stream();
    const uint32_t tmem = ld_smem(slot_addr);
    // this thread's row of the sums: of 64 rows, tensor memory has 16 in each quarter
    const uint32_t mine = P.m == 64 ? lane < 16 ? warp * 16u + lane : 128u : tid, r = r0 + mine;
    float a = 1.0f, bias = 0.0f;

    if (warp == 0) {
        const uint32_t lead = elected();
        uint32_t k = 0, s = 0, phase = 1;
        for (; k < nk; ++k) {
            const uint32_t at = ring + s * P.stage, bar = full + 8 * s, first = (k0 + k) * P.chunk;
            if (k >= P.stages && !bar_wait_warp(empty + 8 * s, phase, abort_word)) break;
            if (first < P.whole) {
                bar_expect_by(bar, P.stage, lead);
                tma_load_3d_by(at + P.chunk * P.x_block, &w_map, 0, int32_t(r0), int32_t(first), bar, lead);
                tma_load_3d_by(at, &x_map, 0, int32_t(t0), int32_t(first), bar, lead);
            } else {
                bar_expect_by(bar, P.w_block + P.x_block, lead);
                tma_load_2d_by(at + P.chunk * P.x_block, &w_tail, int32_t(P.whole * 128u), int32_t(r0), bar, lead);
                tma_load_2d_by(at, &x_tail, int32_t(P.whole * 128u), int32_t(t0), bar, lead);
            }
            if (++s == P.stages) s = 0, phase ^= 1u;
        }
        if (ld_smem(abort_word))                         // nothing may land after the CTA's end
            for (uint32_t j = k > P.stages ? k - P.stages : 0; j < k; ++j) bar_drain(full + 8 * (j % P.stages), (j / P.stages) & 1u);
    } else if (warp == 1) {
        const uint32_t lead = elected(), idesc = i8_idesc(P.m, BN);
        uint32_t s = 0, phase = 0, any = 0;
        for (uint32_t k = 0; k < nk; ++k) {
            if (!bar_wait_warp(full + 8 * s, phase, abort_word)) break;
            tc_after();
            const uint32_t at = ring + s * P.stage, first = (k0 + k) * P.chunk, blocks = first < P.whole ? min(P.chunk, P.whole - first) : 1u;
            uint64_t da = operand_desc(at + P.chunk * P.x_block), db = operand_desc(at);
            for (uint32_t n = 0; n < blocks; ++n, da += P.w_block >> 4, db += P.x_block >> 4) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) mma_i8(tmem, da + 2 * i, db + 2 * i, idesc, any | i, lead);
                any = 1;
            }
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
        T *y = static_cast<T *>(P.y) + int64_t(t0) * P.ldy + r;
#pragma unroll 2
        for (uint32_t c = 0; c < BN && t0 + c < P.T; c += 16)
            put_sixteen<E>(tmem + ((warp * 32u) << 16) + c, scales + 4 * c, y + int64_t(c) * P.ldy, P.ldy, r < r1 ? min(16u, P.T - t0 - c) : 0u, a, bias);
    } else {
        // CTA p finishes tokens p each .. (p + 1) each, of which all send it their sums: a place for each CTA, beside the stages, which others may still be
        // using, four tokens of a row in 16 bytes.  Nobody reads another's memory, so that one barrier is all.
        const uint32_t tokens = min(BN, P.T - t0), each = ((tokens + P.split - 1u) / P.split + 3u) / 4u * 4u, sums = ring + P.sums;
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");                            // (all have begun)
        uint32_t owner = 0, local = 0;
        for (uint32_t c = 0; c < tokens; c += 16) {
            uint32_t v[16];
            tc_load16(tmem + ((warp * 32u) << 16) + c, v);
            tc_loaded16(v);
#pragma unroll
            for (uint32_t i = 0; i < 16; i += 4) {
                if (mine < 128 && c + i < tokens)
                    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.v4.u32 [a], {%2, %3, %4, %5};\n\t}"
                                 ::"r"(sums + ((rank * 128u + mine) * each + local) * 4u), "r"(owner), "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]) : "memory");
                local += 4;
                if (local == each) local = 0, ++owner;
            }
        }
        cluster_sync();
        const uint32_t row = r0 + tid, first = rank * each;
        if (row < r1) {
            if (P.a) a = __ldg(P.a + row);
            if (P.bias) bias = __ldg(P.bias + row);
            T *y = static_cast<T *>(P.y) + int64_t(t0 + first) * P.ldy + row;
#pragma unroll 2
            for (uint32_t q = 0; q < each && first + q < tokens; q += 4) {
                uint4 sum = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (uint32_t p = 0; p < 8; ++p)
                    if (p < P.split) {
                        const uint4 v = ld_smem16(sums + ((p * 128u + tid) * each + q) * 4u);
                        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
                    }
                const uint4 s = ld_smem16(scales + 4 * (first + q));
                const uint32_t n = tokens - first - q;
                y[0] = E::of(scaled(sum.x, __uint_as_float(s.x), a, bias));
                if (n > 1) y[P.ldy] = E::of(scaled(sum.y, __uint_as_float(s.y), a, bias));
                if (n > 2) y[2 * P.ldy] = E::of(scaled(sum.z, __uint_as_float(s.z), a, bias));
                if (n > 3) y[3 * P.ldy] = E::of(scaled(sum.w, __uint_as_float(s.w), a, bias));
                y += 4 * P.ldy;
            }
        }
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

// How strips would share out the work, `split` CTAs to a strip, and an estimate of the time in ns.
struct StripPlan {
    uint32_t split, strips, rows, tokens;        // rows and tokens of a block, in whole eights
    uint64_t grid, ns;
};
StripPlan strip_plan(const ProductParams &P, uint32_t C, uint32_t bn, uint32_t split, uint32_t sms) {
    StripPlan p;
    const uint64_t tiles_t = (P.T + bn - 1u) / bn;
    p.split = split;
    // as many strips as make one CTA on each SM, or a whole number of them where strips of 128 rows are more
    const uint64_t least = (uint64_t(P.R) + 127u) / 128u, round = sms / split / tiles_t;
    uint64_t strips = round ? (least + round - 1u) / round * round : least;
    if (strips > P.R) strips = P.R;
    p.strips = uint32_t(strips);
    p.rows = (uint32_t((P.R + strips - 1u) / strips) + 7u) / 8u * 8u;
    p.tokens = P.T < bn ? (P.T + 7u) / 8u * 8u : bn;
    p.grid = strips * tiles_t * split;
    // A block of columns takes its operands' way from L2, 100 bytes/ns for an SM, or the instructions', (rows + tokens) of 0.8 ns; the weight
    // comes from memory at 6200 bytes/ns; a cluster's join takes 0.9 us and 0.6 ns for each sum of a strip (fitted to 1 - 64 tokens x 64 x 8192 .. 5120 x 17408:
    // 1024 x 8192 with clusters of eight and without 4.6 / 8.4 us for one token, 5.3 / 10.5 for 32, 7.9 / 10.5 for 64).
    const uint64_t block = 8u * ((p.rows <= 64 ? 64u : 128u) + bn) / 10u, way = (p.rows + p.tokens) * 128u / 100u, each = block > way ? block : way;
    const uint64_t rounds = 1u + (p.grid - 1u) / sms, busy = rounds * ((P.blocks + split - 1u) / split) * each;
    const uint64_t memory = uint64_t(P.R) * C / 6200u;
    p.ns = 3300u + (busy > memory ? busy : memory) + (split > 1 ? 900u + uint64_t(p.rows) * P.T * 10u / 17u : 0u);
    return p;
}

template <uint32_t BN, class E>
int launch_strip(ProductParams P, const Operands &o, const StripPlan &plan, uint32_t sms, cudaStream_t st) {
    using G = StripShape<BN>;
    static bool configured[64] = {};
    int rc = op_configure(product_strip_kernel<BN, E>, G::kMost, configured);
    if (rc) return rc;
    if (plan.grid > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    P.split = plan.split;
    P.strips = plan.strips;
    P.m = plan.rows <= 64 ? 64 : 128;
    P.w_block = plan.rows * 128u;
    P.x_block = plan.tokens * 128u;
    const uint32_t block = P.w_block + P.x_block;
    P.whole = o.C / 128u;
    // One CTA to an SM with all of its memory; or two that share it, the next one beginning while the last one ends, where there are more CTAs than SMs or
    // a CTA's share is not much more than fits (4096 x 4096, 1 token: 5.8 us, 6.4 with all memory; 5120 x 17408 19.9, 17.8: the border between the two is known no better than that).
    // (The place of a cluster's sums comes off it.)
    const uint32_t join = plan.split > 1 ? 512u * plan.split * (((plan.tokens + plan.split - 1u) / plan.split + 3u) / 4u * 4u) : 0u, room = (plan.grid > sms || plan.split > 2 || uint64_t(block) * P.blocks / plan.split <= 310u * 1024u ? 92u : 204u) * 1024u - join;
    // Four blocks to a stage where three stages of them fit: a stage costs the issuing warps some 250 cycles, a block's instructions 130
    P.chunk = 4;
    while (P.chunk > 1 && 3 * P.chunk * block > room) P.chunk /= 2;
    P.stage = P.chunk * block;
    P.stages = room / P.stage;
    if (P.stages > G::kMaxStages) P.stages = G::kMaxStages;
    // (the last stage's instructions may read beyond it, into the sums' place or the tail)
    P.sums = P.stages * P.stage + G::kTail;
    const uint32_t smem = G::kSmem(P.stages, P.stage) + join;
    CUtensorMap wm, xm, wt, xt;
    if (P.whole && ((rc = block_map(&wm, o.w, P.whole, P.R, uint64_t(o.ldw), plan.rows, P.chunk)) ||
                    (rc = block_map(&xm, o.x, P.whole, P.T, uint64_t(o.ldx), plan.tokens, P.chunk))))
        return rc;
    if (P.blocks > P.whole) {
        if ((rc = byte_map(&wt, o.w, o.C, P.R, uint64_t(o.ldw), 128, plan.rows, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
        if ((rc = byte_map(&xt, o.x, o.C, P.T, uint64_t(o.ldx), 128, plan.tokens, CU_TENSOR_MAP_SWIZZLE_128B))) return rc;
        if (!P.whole) wm = wt, xm = xt;
    } else wt = wm, xt = xm;                             // (not used)
    return op_launch(product_strip_kernel<BN, E>, uint32_t(plan.grid), 128, smem, plan.split, st, P, wm, xm, wt, xt) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// ---- many tokens: a pair of CTAs per tile -----------------------------------------------------------------------------------
// Two CTAs share tiles of 256 rows of the weight by N tokens (tcgen05 cta_group::2): each has half of the weight's rows and half of the tokens
// in its shared memory, and keeps the sums of its 128 rows with all tokens in its tensor memory, twice, so that a tile is read out while the next one
// is summed.  8192^3 in 334 - 373 us in a short graph of calls (3.0 - 3.3 PFLOP/s; operands from L2 at 12 TB/s), 371 - 434 called one after another, where the power cap lowers the clock; 777 x 3000 x 1744 in 10.1.
//   warp 0        brings the operands in
//   warp 1        of the first CTA issues the products
//   warps 2 - 9   sums to y: two warps to each quarter of the rows, half of the tokens each
template <uint32_t N>
struct PairShape {
    static constexpr uint32_t kA = kBlock * 128, kB = N / 2 * 128, kStage = kA + kB, kStages = N == 256 ? 6 : N == 192 ? 7 : 9;
    static constexpr uint32_t kBars = kStages * kStage, kScales = kBars + 512, kSmem = kScales + 2 * 4 * N + 1024, kCols = N > 128 ? 512 : 256, kThreads = 320;
    static_assert(kSmem <= 232448 && 2 * N <= kCols && kB % 1024 == 0 && N % 32 == 0);
};

template <uint32_t N, class E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairShape<N>::kThreads, 1)
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
        for (uint32_t i = 0; i < 2; ++i) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, 16);
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
    } else if (warp >= 2) {
        const uint32_t quarter = warp & 3u, c0 = warp >= 6 ? N / 2 : 0;
        // (after a wait that ran out the warps still meet at the barrier, tile by tile, and store nothing)
        for (uint32_t tile = pair; tile < tiles; tile += pairs, ++n) {
            const uint32_t r = (tile % P.strips) * 256u + rank * 128u + quarter * 32u + lane, t0 = (tile / P.strips) * N, scales = base + G::kScales + (n & 1u) * 4u * N;
            const float a = P.a && r < P.R ? __ldg(P.a + r) : 1.0f, bias = P.bias && r < P.R ? __ldg(P.bias + r) : 0.0f;
            // (the buffer's last tile but one has been read by all: they have been through the barrier of the last one)
            if (tid - 64u < N) st_smem(scales + 4 * (tid - 64u), __float_as_uint(t0 + tid - 64u < P.T ? __ldg(P.s + t0 + tid - 64u) : 0.0f));
            asm volatile("barrier.sync.aligned 1, 256;" ::: "memory");
            ok = ok && bar_wait_warp(acc_full + 8 * (n & 1u), (n >> 1) & 1u, abort_word);
            if (!ok) continue;
            tc_after();
            T *y = static_cast<T *>(P.y) + int64_t(t0) * P.ldy + r;
#pragma unroll 2
            for (uint32_t c = c0; c < c0 + N / 2 && t0 + c < P.T; c += 16)
                put_sixteen<E>(tmem + (n & 1u) * N + ((quarter * 32u) << 16) + c, scales + 4 * c, y + int64_t(c) * P.ldy, P.ldy, r < P.R ? min(16u, P.T - t0 - c) : 0u, a, bias);
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
    const uint32_t pairs = uint32_t(op_sms()) / 2u;
    if (!pairs) return EP_ERR_CUDA;
    if (tiles > 0x7FFFFFFFu || (tiles / pairs + 1u) * P.blocks > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    const uint32_t grid = 2u * uint32_t(tiles < pairs ? tiles : pairs);
    return op_launch(product_pair_kernel<N, E>, grid, G::kThreads, G::kSmem, 1, st, P, wm, xm) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// Which kernel: the least of the estimates.  Pairs take a round of tiles after another, each a time for a block of columns that grows with the SMs at work as L2
// becomes what bounds it, and a last read-out.  us, strips of 64 / pairs of 128 / 192 / 256 tokens: 128 tokens x 4096^2 8.1 / 9.1 / - / 12.9, 192 x 10240 x 3840 23.2 /
// 16.1 / 13.3 / 14.9, 512 x 1024 x 8192 10.5 / 14.7 / 17.4 / 22.2, x 5120 x 17408 84.6 / 54.1 / 38.5 / 45.6, x 8192^2 47.7 / 32.7 / 34.4 / 26.5, 777 x 3000 x 1744 - /
// 11.7 / 9.7 / 10.7, 8192^3 - / 468 / 389 / 355.
template <class E>
int launch_product(const ProductParams &P, const Operands &o, cudaStream_t st) {
    const uint32_t sms = uint32_t(op_sms()), pairs = sms / 2u;
    if (!pairs) return EP_ERR_CUDA;
    const uint32_t bn = P.T <= 16 ? 16u : P.T <= 32 ? 32u : 64u;
    StripPlan best = strip_plan(P, o.C, bn, 1, sms);
    if (P.T <= 64)                                       // a cluster for each strip; not fewer than four blocks to a CTA
        for (const uint32_t split : {2u, 8u})
            if (P.blocks >= 4u * split) {
                const StripPlan p = strip_plan(P, o.C, bn, split, sms);
                if (p.ns < best.ns && p.grid <= sms) best = p;
            }
    if (P.T > 64) {
        const auto pair_ns = [&](uint32_t n, uint64_t block, uint64_t more, uint64_t end) {
            const uint64_t tiles = uint64_t((P.R + 255u) / 256u) * ((P.T + n - 1u) / n), rounds = (tiles + pairs - 1u) / pairs;
            const uint64_t one = P.blocks * (block + more * (tiles < pairs ? tiles : pairs) / pairs), busy = rounds * (one > end ? one : end);
            const uint64_t memory = uint64_t(P.R) * o.C / 6200u;
            return 3300u + end + (busy > memory ? busy : memory);
        };
        const uint64_t of128 = pair_ns(128, 170, 65, 600), of192 = pair_ns(192, 222, 60, 1200), of256 = pair_ns(256, 275, 55, 1900);
        if (of256 < best.ns && of256 <= of192 && of256 <= of128) return launch_pair<256, E>(P, o, st);
        if (of192 < best.ns && of192 < of128) return launch_pair<192, E>(P, o, st);
        if (of128 < best.ns) return launch_pair<128, E>(P, o, st);
    }
    if (bn == 16) return launch_strip<16, E>(P, o, best, sms, st);
    if (bn == 32) return launch_strip<32, E>(P, o, best, sms, st);
    return launch_strip<64, E>(P, o, best, sms, st);
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
    if (j.d_x == static_cast<const void *>(j.d_q)) return EP_ERR_BAD_ARG;        // (q's rows lie where other rows still have to be read)
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
    P.x_vec = aligned(j.d_x, 16) && P.ldx % 16 == 0 ? 2 : aligned(j.d_x, 8) && P.ldx % 8 == 0 ? 1 : 0;
    P.q_vec = aligned(j.d_q, 8) && j.ldq % 8 == 0 ? 2 : aligned(j.d_q, 4) && j.ldq % 4 == 0 ? 1 : 0;
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
    if (j.d_y == j.d_x || j.d_y == j.d_w) return EP_ERR_BAD_ARG;                 // (every tile reads operands that other tiles' results would lie on)
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
