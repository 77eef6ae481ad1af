// Keys and values in pages of E4M3 with one scale for each page and head: writing new tokens, and the attention that
// reads the pages.
#include "kv_cache.hpp"

#include <algorithm>

using namespace ep;

namespace {

__device__ unsigned int g_cache_status = 0;

// ======================================================================================================================
// Append.  For a page and head with scale s and older tokens q: s' = max(s, the smallest power of two that holds the new tokens), the
// older tokens become e4m3(q s / s') if it grew, the new ones e4m3(x / s').  Powers of two: moving to a larger scale is exact but
// for values that fall below E4M3's normal range, so a token is not rounded again each time its page's scale grows.  A page without
// older tokens forgets what it held.  One warp (or CTA) per page and head, for keys and values together: what bounds a page
// is one chain of reads, lengths, table, rows (with keys and values apart 5 prompts of up to 4096 tokens took 26.4 us, together 23.2); a single new token
// that fits the scale costs one read and write of its row.  Registers allow four CTAs to an SM, each with one page under way: those prompts are 2720
// CTAs, 4.6 rounds of them, at 2.8 TB/s.
// ======================================================================================================================
struct AppendParams {
    Requests q;
    const void *x[2];
    int64_t ldx[2], ldh[2];
    uint8_t *cache[2];
    float *scales[2];
    uint32_t D;
    uint32_t spans;               // grid: spans pages side by side, x heads x requests
};
constexpr uint32_t kLeastScale = 127 - 100;      // of a page of zeros: 2^-100, which any value outgrows

template <class E, uint32_t WARPS>
__global__ void __launch_bounds__(128) append_kernel(const __grid_constant__ AppendParams P) {
    using T = typename E::T;
    // rows of a lane that are held in registers, of keys and values each, and then read once: by a CTA 64 tokens of 128 dimensions, by a warp 16
    constexpr uint32_t kThreads = 32 * WARPS, kHeld = 8;
    __shared__ float largest_of[2][4];
    op_wait_for_stream();
    const uint32_t tid = WARPS == 1 ? threadIdx.x & 31u : threadIdx.x, lane = tid & 31u;
    uint64_t rest = WARPS == 1 ? uint64_t(blockIdx.x) * 4u + (threadIdx.x >> 5) : blockIdx.x;
    const uint32_t span = uint32_t(rest % P.spans); rest /= P.spans;
    const uint32_t h = uint32_t(rest % P.q.H), b = uint32_t(rest / P.q.H);
    if (b >= P.q.B) return;
    const Extent r = extent_of(P.q, b);
    const uint32_t rows = min(r.rows, r.len);             // (more rows than tokens: the first ones have no place)
    if (rows == 0) return;
    const uint32_t first = r.len - rows, lanes = P.D / 8u, at = tid % lanes * 8u, sub = tid / lanes, step = kThreads / lanes;
    for (uint32_t j = (first >> P.q.shift) + span; j <= (r.len - 1u) >> P.q.shift; j += P.spans) {
        const int32_t id = __ldg(P.q.table + int64_t(b) * P.q.ldt + j);
        if (id < 0 || uint32_t(id) >= P.q.pages) {
            if (tid == 0) atomicOr(&g_cache_status, unsigned(kStatusPage));
            continue;
        }
        const uint32_t p0 = j << P.q.shift, lo = max(first, p0), hi = min(r.len, p0 + P.q.page);        // new tokens of this page
        const uint64_t block = uint64_t(uint32_t(id)) * P.q.H + h;
        const bool once = hi - lo <= kHeld * step, older = lo > p0;
        uint4 held[2][kHeld];
        float had[2] = {0.0f, 0.0f}, a[2] = {0.0f, 0.0f};
        if (older) had[0] = P.scales[0][block], had[1] = P.scales[1][block];
        auto source = [&](uint32_t which) { return static_cast<const T *>(P.x[which]) + int64_t(r.row + (r.rows - rows) + lo - first) * P.ldx[which] + int64_t(h) * P.ldh[which] + at; };
        for (uint32_t from = sub; from < hi - lo; from += kHeld * step) {
#pragma unroll
            for (uint32_t which = 0; which < 2; ++which)
#pragma unroll
                for (uint32_t i = 0; i < kHeld; ++i)
                    held[which][i] = from + i * step < hi - lo ? __ldg(reinterpret_cast<const uint4 *>(source(which) + int64_t(from + i * step) * P.ldx[which])) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (uint32_t which = 0; which < 2; ++which)
#pragma unroll
                for (uint32_t i = 0; i < kHeld; ++i) {
                    const uint4 w = held[which][i];
                    const float v[8] = {E::lo(w.x), E::hi(w.x), E::lo(w.y), E::hi(w.y), E::lo(w.z), E::hi(w.z), E::lo(w.w), E::hi(w.w)};
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k)
                        if (fabsf(v[k]) < __uint_as_float(0x7F800000u)) a[which] = fmaxf(a[which], fabsf(v[k]));
                }
        }
#pragma unroll
        for (uint32_t which = 0; which < 2; ++which) a[which] = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a[which])));
        if constexpr (WARPS > 1) {
            if (lane == 0) largest_of[0][tid >> 5] = a[0], largest_of[1][tid >> 5] = a[1];
            __syncthreads();                              // (and everyone has read the old scales)
#pragma unroll
            for (uint32_t i = 0; i < WARPS; ++i) a[0] = fmaxf(a[0], largest_of[0][i]), a[1] = fmaxf(a[1], largest_of[1][i]);
            __syncthreads();
        } else {
            __syncwarp();
        }
#pragma unroll
        for (uint32_t which = 0; which < 2; ++which) {
            uint8_t *dst = P.cache[which] + (block << P.q.shift) * P.D + at;
            const float need = pow2_biased(max(scale_exponent(a[which], kLeastScale), kLeastScale)), scale = fmaxf(need, had[which]);
            if (older && scale > had[which]) {
                const float ratio = __fdiv_rn(had[which], scale);
                for (uint32_t i = sub; i < lo - p0; i += step) {
                    uint2 w = *reinterpret_cast<uint2 *>(dst + i * P.D);
                    auto moved = [&](uint32_t four) {
                        uint32_t l, g;
                        f16x4_of_e4m3x4(four, l, g);
                        return e4m3x2(Fp16::lo(l) * ratio, Fp16::hi(l) * ratio) | e4m3x2(Fp16::lo(g) * ratio, Fp16::hi(g) * ratio) << 16;
                    };
                    w.x = moved(w.x), w.y = moved(w.y);
                    *reinterpret_cast<uint2 *>(dst + i * P.D) = w;
                }
            }
            const bool power = (__float_as_uint(scale) & 0x7FFFFFu) == 0 && scale >= 1e-30f && scale <= 1e30f;
            const float inverse = __fdiv_rn(1.0f, scale);  // exact for a power of two; other scales (a caller's own) are divided by
            for (uint32_t from = sub; from < hi - lo; from += kHeld * step) {
#pragma unroll
                for (uint32_t i = 0; i < kHeld; ++i) {
                    const uint32_t n = from + i * step;
                    if (n >= hi - lo) break;
                    const uint4 w = once ? held[which][i] : __ldg(reinterpret_cast<const uint4 *>(source(which) + int64_t(n) * P.ldx[which]));
                    float v[8] = {E::lo(w.x), E::hi(w.x), E::lo(w.y), E::hi(w.y), E::lo(w.z), E::hi(w.z), E::lo(w.w), E::hi(w.w)};
                    if (power) {
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k) v[k] = fabsf(v[k]) < __uint_as_float(0x7F800000u) ? v[k] * inverse : __uint_as_float(0x7FFFFFFFu);
                    } else {
#pragma unroll 1
                        for (uint32_t k = 0; k < 8; ++k) v[k] = fabsf(v[k]) < __uint_as_float(0x7F800000u) ? __fdiv_rn(v[k], scale) : __uint_as_float(0x7FFFFFFFu);
                    }
                    *reinterpret_cast<uint2 *>(dst + (lo - p0 + n) * P.D) = make_uint2(e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16, e4m3x2(v[4], v[5]) | e4m3x2(v[6], v[7]) << 16);
                }
            }
            if (tid == 0) P.scales[which][block] = scale;
        }
    }
}

// ======================================================================================================================
// Attention.  o = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q . k_j - m), over the tokens that a row sees.
//
// A row is a query and one of the query heads that share a head of the cache; the rows of a request and head make tiles of 8 NT.
// A tile of rows against all tokens of its request is a segment; a segment is cut into units of 256 tokens, the units of all segments form
// one list, and every CTA takes an equal, contiguous share of it, whatever the requests' lengths (they are read on the device: a
// captured launch serves any).  A CTA's warps take tiles of 32 tokens in turn, each with a running maximum and sum of its own and its own ring
// of tiles brought in by the copy engine, so that nothing waits for another warp before the segment's end; there the warps' results
// are joined in shared memory.  What crosses a CTA's share goes through the workspace: a CTA leaves at most two
// pieces there, its first segment's and its last's, and a second launch joins them.
//
// Products are m16n8k16 with binary16 operands (E4M3 converts to binary16 exactly) and tokens, then value columns, along M: a
// handful of rows fills N = 8, where along M they would be half padding, with twice the scores, accumulators and instructions.
// A row of q becomes binary16 times a power of two that puts its largest magnitude at 2^13: exact for binary16 and bfloat16 alike but for elements 2^-27 and
// more below the row's largest, whose rounding is below fp32's own.  A page's value scale is taken into the exponent, t = score +
// log2(v_scale / one page's of the request), and out of the row's sum again.  The reference m of a row moves, and its accumulators with it, only when some t exceeds it by
// more than 8; weights are 2^(t - m + 7): at most 2^15, and down to 2^-21 of what m stands for with 11 bits.  They are rounded to binary16 because that is the
// products' type; the row's sum takes them before.  Off by up to 2^-12 each and at random, they move an output by some 1.4e-4 of itself
// (one request of 200 000 tokens to FP16: 2.2e-4 off the exact result, with weights of 32 bits 2.1e-4).
// ======================================================================================================================
constexpr uint32_t kTile = 32, kUnit = 256;
constexpr float kSlack = 8.0f, kShift = 7.0f;

// where a piece of a segment is left: O, then m and l of each row
template <uint32_t NT, uint32_t D>
constexpr uint32_t kPiece = 8 * NT * (D + 2);
constexpr uint32_t kDescWords = 8;               // per CTA: the segment that it begins and does not end: request, row tile, head, last CTA + 1

template <uint32_t NT, uint32_t D, uint32_t W>
struct AttendShape {
    static constexpr uint32_t kTileBytes = kTile * D, kStage = 2 * kTileBytes;
    static constexpr uint32_t kStages = 24 / W * (128 / D);
    static constexpr uint32_t kRing = kStages * kStage;                                    // per warp
    static constexpr uint32_t kMeta = W * kRing;                                           // scales of the stages' pages: 2 x (key, value)
    static constexpr uint32_t kBars = kMeta + W * kStages * 16;
    static constexpr uint32_t kJoin = kBars + W * kStages * 8;                             // m, l of the warps' rows
    static constexpr uint32_t kNan = kJoin + W * 8 * NT * 8;                               // the first NaN token of each column, then the abort word
    static constexpr uint32_t kPrefix = kNan + D * 4 + 16;
    static constexpr uint32_t kSmem = kPrefix + 4 * (kMaxRequests + 32) + 1024;
    static_assert(8 * NT * D * 4 <= kRing && kSmem <= 232448);
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {       // an 8 x 8 matrix of 16-bit values over the warp
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float log2_fast(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// over the lanes of equal lane % 4
__device__ __forceinline__ float octs_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
    return fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16));
}
__device__ __forceinline__ float octs_sum(float v) {
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
    return v + __shfl_xor_sync(0xFFFFFFFFu, v, 16);
}

__device__ __forceinline__ uint32_t units_of(const Extent &r, uint32_t G, uint32_t H, uint32_t rows_per_tile) {
    const uint32_t tiles = (r.rows * G + rows_per_tile - 1u) / rows_per_tile;
    return tiles * H * max(1u, (r.len + kUnit - 1u) / kUnit);
}
// query i of n sees tokens 0 .. len - n + i
__device__ __forceinline__ uint32_t seen_by(const AttendParams &P, const Extent &r, uint32_t i) {
    return !P.causal ? r.len : r.len + i + 1u > r.rows ? min(r.len, r.len + i + 1u - r.rows) : 0u;
}

template <class E, uint32_t NT, uint32_t D, uint32_t W>
__global__ void __launch_bounds__(32 * W, 1) attend_kernel(const __grid_constant__ AttendParams P, const __grid_constant__ CUtensorMap k_map,
                                                           const __grid_constant__ CUtensorMap v_map) {
    using S = AttendShape<NT, D, W>;
    using T = typename E::T;
    constexpr uint32_t kRows = 8 * NT, kSteps = D / 16, kPer = D / 4;        // k steps of q k^T; elements of a row that a lane of a quad holds
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *gen = raw + (base - smem_u32(raw));
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), quad = lane & 3u, oct = lane >> 2;
    const uint32_t ring = base + warp * S::kRing, bars = base + S::kBars + warp * S::kStages * 8, meta = base + S::kMeta + warp * S::kStages * 16;
    uint32_t *prefix = reinterpret_cast<uint32_t *>(gen + S::kPrefix), *first_nan = reinterpret_cast<uint32_t *>(gen + S::kNan);
    float2 *join = reinterpret_cast<float2 *>(gen + S::kJoin);
    const uint32_t abort_at = base + S::kNan + D * 4;
    if (lane == 0) {
        for (uint32_t i = 0; i < S::kStages; ++i) bar_init(bars + 8 * i, 3);
        bar_init_done();
    }
    if (tid == 0) st_smem(abort_at, 0);
    for (uint32_t i = tid; i < D; i += 32 * W) first_nan[i] = 0xFFFFFFFFu;
    op_wait_for_stream();
    const uint32_t all = prefix_sums(P.q.B, [&](uint32_t i) { return units_of(extent_of(P.q, i), P.G, P.q.H, kRows); }, P.most, prefix, reinterpret_cast<uint32_t *>(join));
    if (all == 0 && blockIdx.x == 0 && tid == 0 && prefix[P.q.B]) atomicOr(&g_cache_status, unsigned(kStatusPage));
    const uint32_t ctas = min(P.grid, all);               // those with a share: none of theirs is empty
    const uint32_t u_begin = blockIdx.x < ctas ? uint32_t(uint64_t(all) * blockIdx.x / ctas) : 0u,
                   u_end = blockIdx.x < ctas ? uint32_t(uint64_t(all) * (blockIdx.x + 1u) / ctas) : 0u;
    uint32_t *desc = P.workspace ? reinterpret_cast<uint32_t *>(P.workspace) + blockIdx.x * kDescWords : nullptr;
    float *pieces = P.workspace ? P.workspace + size_t(P.grid) * kDescWords + size_t(blockIdx.x) * 2u * kPiece<NT, D> : nullptr;
    if (desc && tid == 0) desc[3] = 0;

    uint32_t issued = 0, taken = 0;                       // tiles of this warp's ring
    uint32_t b = 0;
    for (uint32_t u = u_begin; u < u_end;) {
        // ---- the segment of unit u ------------------------------------------------------------------------------------
        b = request_of(prefix, b, P.q.B, u);
        const Extent r = extent_of(P.q, b);
        const uint32_t per_seg = max(1u, (r.len + kUnit - 1u) / kUnit), seg = (u - prefix[b]) / per_seg, first_unit = (u - prefix[b]) % per_seg;
        const uint32_t last_unit = min(per_seg, first_unit + (u_end - u));       // one past the share's last unit of the segment
        const uint32_t h = seg % P.q.H, tile = seg / P.q.H;
        const uint32_t n_rows = r.rows * P.G, row0 = tile * kRows;
        const uint32_t t_begin = first_unit * kUnit, t_end = min(r.len, last_unit * kUnit);
        const uint32_t n_tiles = t_end > t_begin + warp * kTile ? (t_end - t_begin - warp * kTile + W * kTile - 1u) / (W * kTile) : 0u;   // of this warp

        // tile i of this warp begins at token t_begin + (i * W + warp) * 32
        const int32_t *table = P.q.table + int64_t(b) * P.q.ldt;
        const uint32_t per_tile = P.q.page < kTile ? 2u : 1u, box = P.q.page < kTile ? P.q.page : kTile;
        auto page_of = [&](uint32_t i) {                  // lane 0 and 1: the page of the tile's first and second part, -1 if outside
            const uint32_t t = t_begin + (i * W + warp) * kTile + (lane & 1u) * box;
            int32_t id = -1;
            if (i < n_tiles && lane < per_tile && t < r.len) {
                id = __ldg(table + (t >> P.q.shift));
                if (id < 0 || uint32_t(id) >= P.q.pages) {
                    atomicOr(&g_cache_status, unsigned(kStatusPage));
                    id = -1;
                }
            }
            return id;
        };
        auto issue = [&](uint32_t i, int32_t id) {
            const uint32_t s = issued % S::kStages, bar = bars + 8 * s, at = ring + s * S::kStage;
            if (lane == 0) bar_expect(bar, S::kStage);
            __syncwarp();
            if (lane < per_tile) {
                // (a part without a page: rows past the cache's end, which arrive as zeros)
                const uint32_t row = id < 0 ? P.q.pages * P.q.H << P.q.shift : ((uint32_t(id) * P.q.H + h) << P.q.shift) + ((t_begin + (i * W + warp) * kTile) & (P.q.page - 1u));
                tma_load_2d(at + lane * box * D, &k_map, 0, int32_t(row), bar);
                tma_load_2d(at + S::kTileBytes + lane * box * D, &v_map, 0, int32_t(row), bar);
            }
            if (lane < 2) {
                const uint32_t m = meta + s * 16 + lane * 8;
                const int32_t first = __shfl_sync(0x3u, id, 0), mine = per_tile == 2 ? id : first;
                if (mine >= 0) {
                    const size_t block = size_t(uint32_t(mine)) * P.q.H + h;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(m), "l"(P.ks + block) : "memory");
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(m + 4), "l"(P.vs + block) : "memory");
                } else {
                    st_smem(m, 0xBF800000u);              // -1: left out
                    st_smem(m + 4, 0x3F800000u);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
            }
            __syncwarp();
            ++issued;
        };
        const float vs_first = first_scale(P.q, P.vs, b, h, r.len), per_first = __frcp_rn(vs_first);
        int32_t next_page = page_of(0);
        uint32_t asked = 0;
#pragma unroll 1
        for (; asked < min(n_tiles, S::kStages); ++asked) {
            const int32_t id = next_page;
            next_page = page_of(asked + 1);
            issue(asked, id);
        }

        // ---- rows of q as right operands: lane 4 oct + quad holds a quarter of row 8 n + oct, and in the accumulators rows 8 n + 2 quad, + 1 ------
        uint32_t qb[NT][kSteps][2];
        float fac[NT][2];                                 // of a row's scores, without the keys' scale
        uint32_t lim[NT][2];                              // tokens that a row sees
        uint32_t lim_min = 0xFFFFFFFFu, lim_max = 0;
#pragma unroll
        for (uint32_t n = 0; n < NT; ++n) {
            const uint32_t row = row0 + n * 8 + oct, i = row / P.G, g = row % P.G;
            const bool real = row < n_rows;
            uint32_t w[kPer / 2];
            const T *src = static_cast<const T *>(P.x) + int64_t(r.row + i) * P.ldq + int64_t(h * P.G + g) * P.ldqh + quad * kPer;
#pragma unroll
            for (uint32_t c = 0; c < kPer / 8; ++c) {
                const uint4 v = real ? __ldg(reinterpret_cast<const uint4 *>(src) + c) : make_uint4(0, 0, 0, 0);
                w[4 * c] = v.x, w[4 * c + 1] = v.y, w[4 * c + 2] = v.z, w[4 * c + 3] = v.w;
            }
            float a = 0.0f;
#pragma unroll
            for (uint32_t c = 0; c < kPer / 2; ++c) a = max3(a, fabsf(E::lo(w[c])), fabsf(E::hi(w[c])));
            a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
            a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
            // 2^up puts the row's largest magnitude in [2^13, 2^14); a row of zeros or with an infinity stays as it is
            const int32_t ea = int32_t(__float_as_uint(a) >> 23);
            const int32_t up = ea == 0 || ea == 255 ? 0 : min(140 - ea, 100);
            const float mul = pow2_biased(uint32_t(127 + up)), f = P.scale_log2 * pow2_biased(uint32_t(127 - up));
#pragma unroll
            for (uint32_t st = 0; st < kSteps; ++st) {
                qb[n][st][0] = Fp16::two(E::lo(w[2 * st]) * mul, E::hi(w[2 * st]) * mul);
                qb[n][st][1] = Fp16::two(E::lo(w[2 * st + 1]) * mul, E::hi(w[2 * st + 1]) * mul);
            }
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e) {
                fac[n][e] = __shfl_sync(0xFFFFFFFFu, f, int(4u * (2u * quad + e)));
                const uint32_t mine = row0 + n * 8 + 2 * quad + e;
                lim[n][e] = mine < n_rows ? seen_by(P, r, mine / P.G) : 0u;
                lim_max = max(lim_max, lim[n][e]);
                lim_min = min(lim_min, mine < n_rows ? lim[n][e] : 0xFFFFFFFFu);
            }
        }
        lim_min = __reduce_min_sync(0xFFFFFFFFu, lim_min);
        lim_max = __reduce_max_sync(0xFFFFFFFFu, lim_max);

        // o: value columns oct D / 8 + 2 j (and + 1) of rows 8 n + 2 quad, + 1
        float o[D / 16][NT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (uint32_t n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = -INFINITY, l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (uint32_t j = 0; j < D / 16; ++j) o[j][n][0] = o[j][n][1] = o[j][n][2] = o[j][n][3] = 0.0f;
        }

#pragma unroll 1
        for (uint32_t i = 0; i < n_tiles; ++i) {
            const uint32_t s = taken % S::kStages, at = ring + s * S::kStage, t0 = t_begin + (i * W + warp) * kTile;
            const bool ok = bar_wait_warp(bars + 8 * s, (taken / S::kStages) & 1u, abort_at);
            ++taken;
            if (ok && t0 < lim_max) {
                float ks[2], vs[2];
#pragma unroll
                for (uint32_t p = 0; p < 2; ++p) {
                    ks[p] = __uint_as_float(ld_smem(meta + s * 16 + 8 * p));
                    vs[p] = fmaxf(__uint_as_float(ld_smem(meta + s * 16 + 8 * p + 4)) * per_first, kLeastRatio);
                }
                const bool edge = t0 + kTile > lim_min || ks[0] < 0.0f || ks[1] < 0.0f;
                // ---- scores: c0, c1 of m tile x are token t0 + 16 x + oct against rows 8 n + 2 quad, + 1; c2, c3 token + 8 -------
                float sc[2][NT][4];
#pragma unroll
                for (uint32_t x = 0; x < 2; ++x) {
                    uint32_t kw[2][kPer / 4];
#pragma unroll
                    for (uint32_t half = 0; half < 2; ++half)
#pragma unroll
                        for (uint32_t c = 0; c < kPer / 16; ++c) {
                            // 16-byte pieces of a row lie swizzled: of 128 bytes by the row's number mod 8, of 64 by half of it mod 4
                            const uint32_t row = x * 16 + half * 8 + oct, piece = quad * (kPer / 16) + c, sw = D == 128 ? piece ^ (row & 7u) : piece ^ ((row >> 1) & 3u);
                            const uint4 v = ld_smem16(at + row * D + 16 * sw);
                            kw[half][4 * c] = v.x, kw[half][4 * c + 1] = v.y, kw[half][4 * c + 2] = v.z, kw[half][4 * c + 3] = v.w;
                        }
#pragma unroll
                    for (uint32_t n = 0; n < NT; ++n) sc[x][n][0] = sc[x][n][1] = sc[x][n][2] = sc[x][n][3] = 0.0f;
#pragma unroll
                    for (uint32_t st = 0; st < kSteps; ++st) {
                        uint32_t a0, a1, a2, a3;
                        f16x4_of_e4m3x4(kw[0][st], a0, a2);
                        f16x4_of_e4m3x4(kw[1][st], a1, a3);
#pragma unroll
                        for (uint32_t n = 0; n < NT; ++n) mma16816(sc[x][n], a0, a1, a2, a3, qb[n][st][0], qb[n][st][1]);
                    }
                }
                // ---- t = score + log2(v_scale ratio), the reference, weights -------------------------------------------------------------
                const float lift[2] = {log2_fast(vs[0]), log2_fast(vs[1])}, sink[2] = {__frcp_rn(vs[0]), __frcp_rn(vs[1])};
                bool move = false;
#pragma unroll
                for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
                    for (uint32_t x = 0; x < 2; ++x)
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c) {
                            float t = fmaf(sc[x][n][c], fac[n][c & 1u] * ks[x], lift[x]);
                            if (edge && (t0 + x * 16 + oct + (c >> 1) * 8 >= lim[n][c & 1u] || ks[x] < 0.0f)) t = -INFINITY;
                            sc[x][n][c] = t;
                            move |= t > m[n][c & 1u] + kSlack;                    // (also from -infinity)
                        }
                if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
                    for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
                        for (uint32_t e = 0; e < 2; ++e) {
                            const float top = octs_max(fmaxf(fmaxf(sc[0][n][e], sc[0][n][e + 2]), fmaxf(sc[1][n][e], sc[1][n][e + 2])));
                            const float now = fmaxf(m[n][e], top), f = now == -INFINITY ? 1.0f : exp2_fast(m[n][e] - now);
                            m[n][e] = now;
                            l[n][e] *= f;
#pragma unroll
                            for (uint32_t j = 0; j < D / 16; ++j) o[j][n][e] *= f, o[j][n][e + 2] *= f;
                        }
                }
                uint32_t pb[2][NT][2];
#pragma unroll
                for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
                    for (uint32_t x = 0; x < 2; ++x) {
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c) sc[x][n][c] = exp2_fast(sc[x][n][c] - (m[n][c & 1u] == -INFINITY ? 0.0f : m[n][c & 1u] - kShift));
#pragma unroll
                        for (uint32_t e = 0; e < 2; ++e) l[n][e] = fmaf(sc[x][n][e] + sc[x][n][e + 2], sink[x], l[n][e]);
                        // tokens by rows, turned to rows by tokens: the right operand of the second product
                        pb[x][n][0] = transposed(Fp16::two(sc[x][n][0], sc[x][n][1]));
                        pb[x][n][1] = transposed(Fp16::two(sc[x][n][2], sc[x][n][3]));
                    }
                // ---- o += v w: k step x holds tokens t0 + 16 x .. + 15 -----------------------------------------------------------------
#pragma unroll
                for (uint32_t x = 0; x < 2; ++x) {
                    constexpr uint32_t kCols = D / 8;                                    // bytes of a row that a lane takes
                    uint32_t vw[4][kCols / 4];
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) {
                        const uint32_t row = x * 16 + quad * 2 + (j & 1u) + (j >> 1) * 8;
                        if constexpr (D == 128) {
                            const uint4 v = ld_smem16(at + S::kTileBytes + row * D + 16 * (oct ^ (row & 7u)));
                            vw[j][0] = v.x, vw[j][1] = v.y, vw[j][2] = v.z, vw[j][3] = v.w;
                        } else {
                            const uint32_t a = at + S::kTileBytes + row * D + 16 * ((oct >> 1) ^ ((row >> 1) & 3u)) + 8 * (oct & 1u);
                            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(vw[j][0]), "=r"(vw[j][1]) : "r"(a));
                        }
                    }
                    // Where some rows do not see all of the tile's tokens: tokens past the request's end may hold anything and count as zeros, and
                    // a NaN counts for the rows that see its token only (0 * NaN is NaN) - it is taken out here and put into those rows at the end.
                    if (edge)
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) {
                            const uint32_t token = t0 + x * 16 + quad * 2 + (j & 1u) + (j >> 1) * 8;
#pragma unroll
                            for (uint32_t c = 0; c < kCols / 4; ++c) {
                                if (token >= r.len) vw[j][c] = 0;
                                uint32_t is = ((vw[j][c] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                                if (is) {
                                    vw[j][c] &= ~((is >> 7) * 255u);
#pragma unroll 1
                                    for (; is; is &= is - 1u) atomicMin(first_nan + oct * kCols + 4u * c + (uint32_t(__ffs(int(is)) - 1) >> 3), token);
                                }
                            }
                        }
#pragma unroll
                    for (uint32_t c = 0; c < kCols / 4; ++c) {
                        // bytes of two tokens side by side: columns 4 c, 4 c + 1 in the low words, 4 c + 2, 4 c + 3 in the high ones
                        uint32_t lo[4], hi[4];
                        f16x4_of_e4m3x4(__byte_perm(vw[0][c], vw[1][c], 0x5140), lo[0], lo[1]);
                        f16x4_of_e4m3x4(__byte_perm(vw[2][c], vw[3][c], 0x5140), lo[2], lo[3]);
                        f16x4_of_e4m3x4(__byte_perm(vw[0][c], vw[1][c], 0x7362), hi[0], hi[1]);
                        f16x4_of_e4m3x4(__byte_perm(vw[2][c], vw[3][c], 0x7362), hi[2], hi[3]);
#pragma unroll
                        for (uint32_t n = 0; n < NT; ++n) {
                            mma16816(o[2 * c][n], lo[0], lo[1], lo[2], lo[3], pb[x][n][0], pb[x][n][1]);
                            mma16816(o[2 * c + 1][n], hi[0], hi[1], hi[2], hi[3], pb[x][n][0], pb[x][n][1]);
                        }
                    }
                }
            }
            __syncwarp();                                 // the stage has been read
            if (asked < n_tiles) {
                const int32_t id = next_page;
                next_page = page_of(asked + 1);
                issue(asked, id);
                ++asked;
            }
        }

        // ---- the warps' results, joined ------------------------------------------------------------------------------------
        // (this warp's ring is empty: every tile asked for has been taken)
        float *mine = reinterpret_cast<float *>(gen + warp * S::kRing);
#pragma unroll
        for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e) {
                const uint32_t row = n * 8 + 2 * quad + e;
                const float sum = octs_sum(l[n][e]);
                if (oct == 0) join[warp * kRows + row] = make_float2(m[n][e], sum);
#pragma unroll
                for (uint32_t j = 0; j < D / 16; ++j) *reinterpret_cast<float2 *>(mine + row * D + oct * (D / 8) + 2 * j) = make_float2(o[j][n][e], o[j][n][e + 2]);
            }
        __syncthreads();
        const bool whole = first_unit == 0 && last_unit == per_seg;
#pragma unroll 1
        for (uint32_t e = tid; e < kRows * D; e += 32 * W) {
            const uint32_t row = e / D, d = e % D, at = row0 + row, i = at / P.G, g = at % P.G;
            if (at >= n_rows) break;
            float top = -INFINITY;
#pragma unroll
            for (uint32_t w = 0; w < W; ++w) top = fmaxf(top, join[w * kRows + row].x);
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f, acc = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < W; ++w) {
                const float2 j = join[w * kRows + row];
                const float f = exp2_fast(j.x - ref);
                sum = fmaf(f, j.y, sum);
                acc = fmaf(f, *reinterpret_cast<const float *>(gen + w * S::kRing + (row * D + d) * 4), acc);
            }
            if (first_nan[d] < seen_by(P, r, i)) acc = __uint_as_float(0x7FFFFFFFu);
            if (whole) {
                const int64_t t = int64_t(r.row + i), head = int64_t(h * P.G + g);
                static_cast<T *>(P.o)[t * P.ldo + head * P.ldoh + d] = E::of(sum == 0.0f ? 0.0f : __fdiv_rn(acc, sum) * vs_first);
                if (P.lse && d == 0) P.lse[t * P.Hq + head] = sum == 0.0f ? -INFINITY : (top - kShift + log2f(sum)) * 0.69314718055994531f;
            } else {
                float *piece = pieces + (u == u_begin ? 0u : kPiece<NT, D>);
                piece[row * D + d] = acc * vs_first;
                if (d == 0) piece[kRows * D + row] = top, piece[kRows * D + kRows + row] = sum;
            }
        }
        if (!whole && first_unit == 0 && tid == 0) {      // this CTA begins the segment: the second launch joins it from here
            const uint32_t end = prefix[b] + (seg + 1u) * per_seg;                       // the segment's end in the list
            uint32_t cta = uint32_t(uint64_t(end - 1u) * ctas / all);                    // the CTA that has its last unit
            while (uint64_t(all) * (cta + 1u) / ctas < end) ++cta;
            while (uint64_t(all) * cta / ctas >= end) --cta;
            desc[0] = b, desc[1] = tile, desc[2] = h, desc[3] = cta + 1u, desc[4] = u == u_begin ? 0u : 1u;
        }
        // the rings are written by the copy engine next: the reads and writes above come first
        fence_proxy_async();
        __syncthreads();
        for (uint32_t i = tid; i < D; i += 32 * W) first_nan[i] = 0xFFFFFFFFu;
        if (u + last_unit - first_unit < u_end) __syncthreads();
        u += last_unit - first_unit;
    }
    if (tid == 0 && ld_smem(abort_at)) atomicOr(&g_cache_status, unsigned(kStatusWait));
    if (ld_smem(abort_at) && lane == 0)                   // (a wait ran out: what is still under way gets its time)
        for (uint32_t j = issued > S::kStages ? issued - S::kStages : 0u; j < issued; ++j) bar_drain(bars + 8 * (j % S::kStages), (j / S::kStages) & 1u);
}

// The segments that cross a share: CTA column k takes the one that CTA k of the first launch began, a CTA for each row.  Its other pieces are
// the first ones of the CTAs after it.  A long request's segment is 40 pieces: their maxima and sums are taken by a thread each, their
// values by two or four threads for each column (a thread per column, piece after piece: 13 us of the 53 that one request of 200 000 tokens took).
constexpr uint32_t kJoinThreads = 256, kMostPieces = 256;
template <class E, uint32_t NT, uint32_t D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendParams P) {
    using T = typename E::T;
    constexpr uint32_t kRows = 8 * NT, kParts = kJoinThreads / D;
    __shared__ float weight[kMostPieces], warp_top[kJoinThreads / 32], warp_sum[kJoinThreads / 32], part_of[kJoinThreads];
    op_wait_for_stream();
    const uint32_t *desc = reinterpret_cast<const uint32_t *>(P.workspace) + blockIdx.x * kDescWords;
    const uint32_t end = desc[3];
    if (end == 0) return;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, n = end - blockIdx.x;       // pieces; at most one per CTA of the first launch
    const uint32_t b = desc[0], tile = desc[1], h = desc[2];
    const Extent r = extent_of(P.q, b);
    const float *all = P.workspace + size_t(P.grid) * kDescWords;
    const uint32_t own = desc[4];
    auto piece = [&](uint32_t c) { return all + (size_t(blockIdx.x + c) * 2u + (c ? 0u : own)) * kPiece<NT, D>; };
    const uint32_t row = blockIdx.y;
    const uint32_t at = tile * kRows + row, i = at / P.G, g = at % P.G;
    if (at >= r.rows * P.G) return;
    const float m = tid < n ? piece(tid)[kRows * D + row] : -INFINITY, l = tid < n ? piece(tid)[kRows * D + kRows + row] : 0.0f;
    float top = m;
#pragma unroll
    for (uint32_t k = 1; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
    if (lane == 0) warp_top[warp] = top;
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kJoinThreads / 32; ++k) top = fmaxf(top, warp_top[k]);
    const float f = tid < n ? exp2_fast(m - (top == -INFINITY ? 0.0f : top)) : 0.0f;
    weight[tid] = f;
    float sum = tid < n ? l * f : 0.0f;
#pragma unroll
    for (uint32_t k = 1; k < 32; k <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
    if (lane == 0) warp_sum[warp] = sum;
    __syncthreads();
    const uint32_t d = tid % D, part = tid / D;
    float acc = 0.0f;
#pragma unroll 8
    for (uint32_t c = part; c < n; c += kParts) acc = fmaf(weight[c], piece(c)[row * D + d], acc);
    part_of[tid] = acc;
    __syncthreads();
    if (part == 0) {
        sum = 0.0f;
#pragma unroll
        for (uint32_t k = 0; k < kJoinThreads / 32; ++k) sum += warp_sum[k];
#pragma unroll
        for (uint32_t k = 1; k < kParts; ++k) acc += part_of[k * D + d];
        const int64_t t = int64_t(r.row + i), head = int64_t(h * P.G + g);
        static_cast<T *>(P.o)[t * P.ldo + head * P.ldoh + d] = E::of(sum == 0.0f ? 0.0f : __fdiv_rn(acc, sum));
        if (P.lse && d == 0) P.lse[t * P.Hq + head] = sum == 0.0f ? -INFINITY : (top - kShift + log2f(sum)) * 0.69314718055994531f;
    }
}

const bool registered = ep::add_status_word([] { return op_status(g_cache_status); });

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

// what both entry points check of the cache and the requests; fills q
int check_cache(const ep_cache &c, const ep_requests &r, Requests &q) {
    if (!c.d_k || !c.d_v || !c.d_k_scales || !c.d_v_scales || !r.d_table || !r.d_seq_lens || !r.d_starts) return EP_ERR_BAD_ARG;
    if (c.pages == 0 || c.heads == 0 || r.columns == 0 || r.ldt < int64_t(r.columns) || r.N > 0x7FFFFFFFu) return EP_ERR_BAD_ARG;
    if (!aligned(c.d_k, 16) || !aligned(c.d_v, 16) || !aligned(c.d_k_scales, 4) || !aligned(c.d_v_scales, 4) || !aligned(r.d_table, 4) ||
        !aligned(r.d_seq_lens, 4) || !aligned(r.d_starts, 4))
        return EP_ERR_BAD_ARG;
    if (c.page < 16 || c.page > 256 || (c.page & (c.page - 1u)) || (c.dim != 64 && c.dim != 128)) return EP_ERR_UNSUPPORTED;
    if (c.pages >= (1u << 27) || c.heads >= (1u << 16) || uint64_t(c.pages) * c.heads * c.page >= (1ull << 31) - 256u || uint64_t(r.columns) * c.page >= (1ull << 31))
        return EP_ERR_UNSUPPORTED;
    q.table = r.d_table;
    q.seq_lens = r.d_seq_lens;
    q.starts = r.d_starts;
    q.ldt = r.ldt;
    q.B = r.B;
    q.N = r.N;
    q.columns = r.columns;
    q.pages = c.pages;
    q.page = c.page;
    q.shift = 0;
    while ((1u << q.shift) < c.page) ++q.shift;
    q.H = c.heads;
    return EP_OK;
}

template <class E>
int launch_append(const AppendParams &P, cudaStream_t st) {
    // a CTA for each page and head where there are more values than a warp holds, else a warp (100 requests of 125 tokens, pages of 16 x 64: 44.9 -> 25.5 us)
    const uint64_t units = uint64_t(P.spans) * P.q.H * P.q.B, average = (uint64_t(P.q.N) + P.q.B - 1u) / P.q.B;
    const bool wide = std::min<uint64_t>(average, P.q.page) * P.D > 2048u;
    const uint64_t grid = wide ? units : (units + 3u) / 4u;
    if (grid > 0x7FFFFFFFu) return EP_ERR_UNSUPPORTED;
    const cudaError_t e = wide ? op_launch(append_kernel<E, 4>, uint32_t(grid), 128, 0, 1, st, P) : op_launch(append_kernel<E, 1>, uint32_t(grid), 128, 0, 1, st, P);
    return e == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

// tiles of eight rows that a warp takes together: one, or two where requests of average size have more rows than that
uint32_t row_tiles(uint32_t N, uint32_t G, uint32_t B) { return uint64_t(N) * G <= 8ull * B ? 1u : 2u; }

template <class E, uint32_t NT, uint32_t D>
int launch_attend(AttendParams P, const ep_cache &c, size_t workspace_bytes, cudaStream_t st) {
    // what registers allow: twelve warps with eight rows (64 requests 211 us, with eight warps 235), eight with sixteen
    constexpr uint32_t W = NT == 1 ? 12 : 8;
    using S = AttendShape<NT, D, W>;
    static bool configured[64] = {};
    int rc = op_configure(attend_kernel<E, NT, D, W>, S::kSmem, configured);
    if (rc) return rc;
    CUtensorMap km, vm;
    const uint64_t rows = uint64_t(c.pages) * c.heads * c.page;
    const CUtensorMapSwizzle sw = D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    const uint32_t box = c.page < kTile ? c.page : kTile;
    if ((rc = byte_map(&km, c.d_k, D, rows, D, D, box, sw)) || (rc = byte_map(&vm, c.d_v, D, rows, D, D, box, sw))) return rc;
    const bool joined = uint64_t(P.q.columns) * c.page > kUnit;             // else a segment is one unit and crosses no share
    if (joined) {
        const size_t need = size_t(P.grid) * (kDescWords + 2u * kPiece<NT, D>) * 4u;
        if (!P.workspace || workspace_bytes < need || !aligned(P.workspace, 16)) return EP_ERR_SCRATCH;
    } else {
        P.workspace = nullptr;
    }
    if (op_launch(attend_kernel<E, NT, D, W>, P.grid, 32 * W, S::kSmem, 1, st, P, km, vm) != cudaSuccess) return EP_ERR_CUDA;
    if (joined && op_launch(join_kernel<E, NT, D>, dim3(P.grid, 8 * NT), kJoinThreads, 0, 1, st, P) != cudaSuccess) return EP_ERR_CUDA;
    return EP_OK;
}

template <class E>
int launch_attend(const AttendParams &P, const ep_cache &c, size_t workspace_bytes, cudaStream_t st) {
    if (row_tiles(P.q.N, P.G, P.q.B) == 1)
        return c.dim == 64 ? launch_attend<E, 1, 64>(P, c, workspace_bytes, st) : launch_attend<E, 1, 128>(P, c, workspace_bytes, st);
    return c.dim == 64 ? launch_attend<E, 2, 64>(P, c, workspace_bytes, st) : launch_attend<E, 2, 128>(P, c, workspace_bytes, st);
}

}  // namespace

extern "C" int ep_cache_append(const ep_append_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_append_job &j = *job;
    const uint32_t B = j.requests.B, N = j.requests.N;
    if (B == 0 || N == 0) return EP_OK;
    AppendParams P;
    std::memset(&P, 0, sizeof(P));
    const int rc = check_cache(j.cache, j.requests, P.q);
    if (rc) return rc;
    if (!j.d_k || !j.d_v || (j.dtype != EP_BF16 && j.dtype != EP_FP16)) return EP_ERR_BAD_ARG;
    if (!aligned(j.d_k, 16) || !aligned(j.d_v, 16) || j.ldk % 8 || j.ldk_head % 8 || j.ldv % 8 || j.ldv_head % 8) return EP_ERR_UNSUPPORTED;
    P.x[0] = j.d_k, P.x[1] = j.d_v;
    P.ldx[0] = j.ldk, P.ldx[1] = j.ldv;
    P.ldh[0] = j.ldk_head, P.ldh[1] = j.ldv_head;
    P.cache[0] = static_cast<uint8_t *>(j.cache.d_k), P.cache[1] = static_cast<uint8_t *>(j.cache.d_v);
    P.scales[0] = j.cache.d_k_scales, P.scales[1] = j.cache.d_v_scales;
    P.D = j.cache.dim;
    // as many pages side by side as a request of twice the average length touches; a longer one's take turns
    const uint64_t average = (uint64_t(N) + B - 1u) / B, most = uint64_t(N) / j.cache.page + 2u;
    P.spans = uint32_t(average > 1 ? std::min<uint64_t>(std::min<uint64_t>(most, j.requests.columns), (2u * average - 1u) / j.cache.page + 2u) : 1u);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return j.dtype == EP_BF16 ? launch_append<Bf16>(P, st) : launch_append<Fp16>(P, st);
}

extern "C" size_t ep_cache_attention_workspace_bytes(uint32_t N, uint32_t B, uint32_t q_heads, uint32_t heads, uint32_t dim) {
    const int n_sms = op_sms();
    if (n_sms <= 0 || heads == 0 || B == 0) return 0;
    const uint32_t sms = std::min(uint32_t(n_sms), kMostPieces);
    if (prompts_serve(N, B, q_heads / heads)) return prompts_workspace_bytes(sms, dim);
    const uint32_t rows = 8u * row_tiles(N, q_heads / heads, B);
    return size_t(sms) * (kDescWords + 2u * rows * (size_t(dim) + 2u)) * 4u;
}

extern "C" int ep_cache_attention(const ep_attention_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_attention_job &j = *job;
    const ep_cache &c = j.cache;
    const uint32_t B = j.requests.B, N = j.requests.N;
    if (B == 0 || N == 0) return EP_OK;
    AttendParams P;
    std::memset(&P, 0, sizeof(P));
    const int rc = check_cache(c, j.requests, P.q);
    if (rc) return rc;
    if (!j.d_q || !j.d_o || (j.dtype != EP_BF16 && j.dtype != EP_FP16) || j.q_heads == 0 || j.q_heads % c.heads || (j.d_lse && !aligned(j.d_lse, 4))) return EP_ERR_BAD_ARG;
    if (!aligned(j.d_q, 16) || j.ldq % 8 || j.ldq_head % 8 || !aligned(j.d_o, 16) || j.ldo % 8 || j.ldo_head % 8 || B > kMaxRequests) return EP_ERR_UNSUPPORTED;
    P.x = j.d_q;
    P.o = j.d_o;
    P.lse = j.d_lse;
    P.ks = c.d_k_scales;
    P.vs = c.d_v_scales;
    P.ldq = j.ldq;
    P.ldqh = j.ldq_head;
    P.ldo = j.ldo;
    P.ldoh = j.ldo_head;
    P.Hq = j.q_heads;
    P.G = j.q_heads / c.heads;
    P.scale_log2 = j.scale * 1.4426950408889634f;
    P.causal = j.causal ? 1u : 0u;
    P.workspace = static_cast<float *>(j.d_workspace);
    // units (of 256 tokens here, of 128 for prompts) are counted in 32 bits; their number can pass 64 on the way
    if (uint64_t(N) * P.G >= (1ull << 31)) return EP_ERR_UNSUPPORTED;
    const uint64_t rows = 8u * row_tiles(N, P.G, B), per_head = ((uint64_t(P.q.columns) * c.page + kUnit - 1u) / kUnit) * ((uint64_t(N) * P.G + rows - 1u) / rows + B), units = per_head * c.heads;
    if (per_head >= (1ull << 30) || units >= (1ull << 30)) return EP_ERR_UNSUPPORTED;
    const int sms = op_sms();
    if (sms <= 0) return EP_ERR_CUDA;
    P.grid = std::min(uint32_t(sms), kMostPieces);
    // of prompts: row tiles of 256, in each at most three places more than tiles of 128 tokens; below 2^32, as N * G > 16 B there
    P.most = prompts_serve(N, B, P.G) ? uint32_t(((uint64_t(P.q.columns) * c.page + 127u) / 128u + 3u) * (uint64_t(N) * P.G / 256u + B) * c.heads) : uint32_t(units);
    P.k = static_cast<const uint8_t *>(c.d_k);
    P.v = static_cast<const uint8_t *>(c.d_v);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (prompts_serve(N, B, P.G)) return launch_prompts(P, j.workspace_bytes, uint64_t(P.q.columns) * c.page > kUnit, c.dim, j.dtype, st);
    return j.dtype == EP_BF16 ? launch_attend<Bf16>(P, c, j.workspace_bytes, st) : launch_attend<Fp16>(P, c, j.workspace_bytes, st);
}
