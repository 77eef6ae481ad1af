// Attention over the paged cache for many rows per request: prompts, and pieces of them.
#include "kv_cache.hpp"

using namespace ep;

namespace {

__device__ unsigned int g_prompts_status = 0;

// ======================================================================================================================
// A unit is 256 rows (a row = a query and one of the query heads that share a head of the cache) of one request and head, as two tiles
// of 128, against the request's tokens, 128 at a time.  Bound by the tensor cores: 2 * 2 * 256 * 128 * D operations for each 128 tokens, in
// binary16, and next to them by the 256 * 128 exponentials (at 16 per cycle and SM as long as the products with D = 128).
//   warps 0 - 3, 4 - 7   a tile's softmax: a thread has a row.  Scores come from tensor memory, the weights go back there (binary16, over
//                        the scores) as the second product's left operand.
//   warps 8 - 11         bring keys and values in and turn them into binary16, exactly, in the layout of the products' right operands; the
//                        work for a token is shared by 256 rows.
//   warp 12              issues the products.  While one tile's softmax runs, the other's products do.
// (Warps 13 - 15 have nothing to do: registers go from one group of four warps to another.)
// The running maximum is a reference m: it moves, and the accumulator in tensor memory is scaled, only when a score exceeds it by more
// than 2^8; weights are 2^(t - m + 7), so at most 2^15, inside binary16.  A page's value scale is taken into
// the exponent, t = score + log2(v_scale), and out of the row's sum again.
// ======================================================================================================================
constexpr uint32_t kUnitRows = 256, kKeys = 128, kThreads = 32 * 16, kNanUnits = 8;
constexpr float kSlack = 8.0f, kShift = 7.0f;

template <uint32_t D>
struct PromptShape {
    static constexpr uint32_t kHalves = D / 64, kHalf = 128 * 128, kTile = kHalves * kHalf;     // 128 rows x D binary16: blocks of 64 columns, 128-byte rows
    static constexpr uint32_t kQ = 0, kK = 2 * kTile, kV = kK + 2 * kTile;
    static constexpr uint32_t kMeta = kV + 2 * kTile;                  // four slots of eight groups of 16 tokens: key scale, log2 value scale, its inverse
    static constexpr uint32_t kNan = kMeta + 4 * 8 * 16;               // some units' first NaN token of each column, then their flags
    static constexpr uint32_t kBars = kNan + kNanUnits * (D + 1) * 4;
    static constexpr uint32_t kPart = kBars + 256, kPrefix = kPart + 128;
    static constexpr uint32_t kSmem = kPrefix + 4 * (kMaxRequests + 32) + 1024;
    static_assert(kSmem <= 232448);
};

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// binary16 x binary16 to fp32, M = 128, N = n; `mn` = the right operand is MN-major
__host__ __device__ constexpr uint32_t f16_idesc(uint32_t n, uint32_t mn) { return (1u << 4) | (mn << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

struct Unit {
    uint32_t b, h, row0;          // request, head of the cache, first of its rows
    Extent r;
    uint32_t n_rows;              // rows of the request
    uint32_t least, most;         // tokens that the unit's first and last rows see
};
__device__ __forceinline__ uint32_t sees(const AttendParams &P, const Extent &r, uint32_t query) {
    return !P.causal ? r.len : r.len + query + 1u > r.rows ? min(r.len, r.len + query + 1u - r.rows) : 0u;
}
__device__ __forceinline__ Unit unit_of(const AttendParams &P, const uint32_t *prefix, uint32_t u) {
    Unit x;
    x.b = request_of(prefix, 0, P.q.B, u);
    const uint32_t rest = u - prefix[x.b];
    x.h = rest % P.q.H;
    x.row0 = rest / P.q.H * kUnitRows;
    x.r = extent_of(P.q, x.b);
    x.n_rows = x.r.rows * P.G;
    x.least = sees(P, x.r, x.row0 / P.G);
    x.most = sees(P, x.r, (min(x.row0 + kUnitRows, x.n_rows) - 1u) / P.G);
    return x;
}

template <class E, uint32_t D>
__global__ void __launch_bounds__(kThreads, 1) prompts_kernel(const __grid_constant__ AttendParams P) {
    using S = PromptShape<D>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *gen = raw + (base - smem_u32(raw));
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    uint32_t *prefix = reinterpret_cast<uint32_t *>(gen + S::kPrefix), *nan_at = reinterpret_cast<uint32_t *>(gen + S::kNan);
    const uint32_t bars = base + S::kBars, k_full = bars, k_free = bars + 16, v_full = bars + 32, v_free = bars + 48, s_full = bars + 64, p_ready = bars + 80,
                   q_ready = bars + 96, o_full = bars + 112, drained = bars + 128, slot_addr = bars + 136, abort_word = bars + 140;
    if (tid == 0) {
        for (uint32_t i = 0; i < 2; ++i) {
            bar_init(k_full + 8 * i, 128), bar_init(v_full + 8 * i, 128);
            bar_init(k_free + 8 * i, 1), bar_init(v_free + 8 * i, 1), bar_init(s_full + 8 * i, 1), bar_init(o_full + 8 * i, 1);
            bar_init(p_ready + 8 * i, 128), bar_init(q_ready + 8 * i, 128);
        }
        bar_init(drained, 1);
        st_smem(abort_word, 0);
        bar_init_done();
    }
    for (uint32_t i = tid; i < kNanUnits * (D + 1); i += kThreads) nan_at[i] = i < kNanUnits * D ? 0xFFFFFFFFu : 0u;
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    op_wait_for_stream();
    const uint32_t tmem = ld_smem(slot_addr);
    const uint32_t all = prefix_sums(P.q.B, [&](uint32_t b) { return (extent_of(P.q, b).rows * P.G + kUnitRows - 1u) / kUnitRows * P.q.H; }, prefix,
                                     reinterpret_cast<uint32_t *>(gen + S::kPart));
    // tensor memory: scores (and weights) of the two tiles, then their accumulators
    const uint32_t s_col[2] = {tmem, tmem + 128u}, o_col[2] = {tmem + 256u, tmem + 384u};
    uint32_t it = 0, n_unit = 0;                          // tiles of tokens and units so far
    bool ok = true;

    // units from the last one on: a request's last rows see the most tokens, and the longest units come first
    // registers: 512 threads x 128 at launch = 128 x (168 + 168 + 104 + 72)
    if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ---- products -----------------------------------------------------------------------------------------------------
        if (warp == 12 && lane == 0) {
            constexpr uint32_t kScores = f16_idesc(kKeys, 0), kValues = f16_idesc(D, 1);
            auto scores = [&](uint32_t t, uint32_t stage) {
#pragma unroll
                for (uint32_t k = 0; k < D / 16; ++k) {
                    const uint32_t at = k / 4 * S::kHalf + k % 4 * 32;
                    mma_f16_ss(s_col[t], operand_desc(base + S::kQ + t * S::kTile + at), operand_desc(base + S::kK + stage * S::kTile + at), kScores, k ? 1u : 0u);
                }
            };
            auto values = [&](uint32_t t, uint32_t stage, uint32_t accumulate) {
#pragma unroll
                for (uint32_t k = 0; k < kKeys / 16; ++k)
                    mma_f16_ts(o_col[t], s_col[t] + 8 * k, operand_desc(base + S::kV + stage * S::kTile + k * 2048, S::kHalf), kValues, accumulate | (k ? 1u : 0u));
            };
            for (uint32_t u = blockIdx.x; u < all && ok; u += gridDim.x) {
                const Unit x = unit_of(P, prefix, all - 1u - u);
                const uint32_t tiles = (x.most + kKeys - 1u) / kKeys;
                if (tiles == 0) continue;
                for (uint32_t i = 0; i < tiles && ok; ++i, ++it) {
                    const uint32_t stage = it & 1u, turn = (it >> 1) & 1u, before = it - 1u;
                    ok = bar_wait(k_full + 8 * stage, turn, abort_word) && (i || bar_wait(q_ready, n_unit & 1u, abort_word));
                    if (!ok) break;
                    tc_after();
                    scores(0, stage);
                    tc_commit(s_full);
                    if (i) {
                        ok = bar_wait(p_ready + 8, before & 1u, abort_word);
                        if (!ok) break;
                        tc_after();
                        values(1, before & 1u, i > 1u);
                        tc_commit(v_free + 8 * (before & 1u));
                    } else {
                        ok = bar_wait(q_ready + 8, n_unit & 1u, abort_word);
                        if (!ok) break;
                        tc_after();
                    }
                    scores(1, stage);
                    tc_commit(s_full + 8);
                    tc_commit(k_free + 8 * stage);
                    ok = bar_wait(v_full + 8 * stage, turn, abort_word) && bar_wait(p_ready, it & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    values(0, stage, i ? 1u : 0u);
                    if (i + 1u == tiles) tc_commit(o_full);
                }
                if (!ok) break;
                const uint32_t before = it - 1u;
                ok = bar_wait(p_ready + 8, before & 1u, abort_word);
                if (!ok) break;
                tc_after();
                values(1, before & 1u, tiles > 1u);
                tc_commit(v_free + 8 * (before & 1u));
                tc_commit(o_full + 8);
                ++n_unit;
            }
            tc_commit(drained);
            bar_drain(drained, 0);                        // nothing is in flight when tensor memory is given back
        }
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        // ---- keys and values ----------------------------------------------------------------------------------------------
        constexpr uint32_t kLanes = D / 16, kPer = 32 / kLanes, kLoads = 32 / kPer;          // lanes of a token; tokens of a load; loads of a warp's 32 tokens
        const uint32_t w = warp - 8u, l = tid - 256u, piece = lane % kLanes, half = piece >> 2;
        for (uint32_t u = blockIdx.x; u < all && ok; u += gridDim.x) {
            const Unit x = unit_of(P, prefix, all - 1u - u);
            const uint32_t tiles = (x.most + kKeys - 1u) / kKeys;
            if (tiles == 0) continue;
            const int32_t *table = P.q.table + int64_t(x.b) * P.q.ldt;
            // The record of NaN two units on is cleared here.  These warps run at most two tiles ahead of the products, so the unit that
            // used it six units ago has long been written; and a warp that is at that unit's first tile has seen a stage freed
            // that all of them filled after this.
            uint32_t *first_nan = nan_at + n_unit % kNanUnits * D, *has_nan = nan_at + kNanUnits * D + n_unit % kNanUnits;
            if (n_unit + 2u >= kNanUnits) {
                if (l < D) nan_at[(n_unit + 2u) % kNanUnits * D + l] = 0xFFFFFFFFu;
                if (l == 0) nan_at[kNanUnits * D + (n_unit + 2u) % kNanUnits] = 0;
            }
            auto page_at = [&](uint32_t t) {              // the page of token t, -1 if there is none
                if (t >= x.r.len) return -1;
                const int32_t id = __ldg(table + (t >> P.q.shift));
                if (id >= 0 && uint32_t(id) < P.q.pages) return id;
                atomicOr(&g_prompts_status, 2u);
                return -1;
            };
            auto load = [&](const uint8_t *cache, uint32_t t0, int32_t id, uint4 (&v)[kLoads]) {
#pragma unroll
                for (uint32_t j = 0; j < kLoads; ++j) {
                    const uint32_t sub = j * kPer + lane / kLanes, t = t0 + w * 32u + sub;
                    const int32_t page = __shfl_sync(0xFFFFFFFFu, id, sub);
                    v[j] = make_uint4(0, 0, 0, 0);
                    if (page >= 0) {
                        const uint8_t *src = cache + (((uint64_t(uint32_t(page)) * P.q.H + x.h) << P.q.shift) + (t & (P.q.page - 1u))) * D + piece * 16u;
                        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[j].x), "=r"(v[j].y), "=r"(v[j].z), "=r"(v[j].w) : "l"(src));
                    }
                }
            };
            // 16 values of a token: two 16-byte pieces of its row in the block of 64 columns; the two halves of a row write
            // them in opposite order, to different banks
            auto store = [&](uint32_t at, const uint4 (&v)[kLoads]) {
#pragma unroll
                for (uint32_t j = 0; j < kLoads; ++j) {
                    const uint32_t row = w * 32u + j * kPer + lane / kLanes;
                    uint32_t f[8];
                    f16x4_of_e4m3x4(v[j].x, f[0], f[1]);
                    f16x4_of_e4m3x4(v[j].y, f[2], f[3]);
                    f16x4_of_e4m3x4(v[j].z, f[4], f[5]);
                    f16x4_of_e4m3x4(v[j].w, f[6], f[7]);
                    const uint32_t to = at + half * S::kHalf + row * 128u, c = 2u * (piece & 3u), sw = row & 7u;
                    const uint32_t a0 = to + ((c ^ sw) << 4), a1 = to + (((c + 1u) ^ sw) << 4);
                    const bool flip = half != 0;
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(flip ? a1 : a0), "r"(flip ? f[4] : f[0]), "r"(flip ? f[5] : f[1]), "r"(flip ? f[6] : f[2]), "r"(flip ? f[7] : f[3]) : "memory");
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(flip ? a0 : a1), "r"(flip ? f[0] : f[4]), "r"(flip ? f[1] : f[5]), "r"(flip ? f[2] : f[6]), "r"(flip ? f[3] : f[7]) : "memory");
                }
                fence_proxy_async();
            };
            // a group's scales (threads 0 - 7), a tile ahead
            float ks = -1.0f, vs = 1.0f;
            auto scales_of = [&](uint32_t t0) {
                if (l >= 8) return;
                const int32_t page = page_at(t0 + 16u * l);
                ks = -1.0f, vs = 1.0f;
                if (page >= 0) {
                    const size_t block = size_t(uint32_t(page)) * P.q.H + x.h;
                    ks = __ldg(P.ks + block), vs = __ldg(P.vs + block);
                }
            };
            uint4 kv[kLoads], vv[kLoads];
            int32_t id = page_at(w * 32u + lane), id_next;
            load(P.k, 0, id, kv);
            scales_of(0);
            for (uint32_t i = 0; i < tiles; ++i, ++it) {
                const uint32_t stage = it & 1u, turn = (it >> 1) & 1u, t0 = i * kKeys;
                load(P.v, t0, id, vv);
                id_next = i + 1u < tiles ? page_at(t0 + kKeys + w * 32u + lane) : -1;
                if (it > 1u) ok = __all_sync(0xFFFFFFFFu, bar_wait(k_free + 8 * stage, turn ^ 1u, abort_word));
                if (!ok) break;
                store(base + S::kK + stage * S::kTile, kv);
                if (l < 8) {
                    const float some = fmaxf(vs, 1e-30f);
                    *reinterpret_cast<float4 *>(gen + S::kMeta + ((it & 3u) * 8u + l) * 16u) = make_float4(ks, log2f(some), __fdiv_rn(1.0f, some), 0.0f);
                }
                bar_arrive(k_full + 8 * stage);
                if (i + 1u < tiles) {
                    load(P.k, t0 + kKeys, id_next, kv);
                    scales_of(t0 + kKeys);
                }
                // a NaN counts for the rows that see its token and no others: where some do not, it is taken out here and put into
                // those rows at the unit's end
                if (t0 + kKeys > x.least) {
#pragma unroll
                    for (uint32_t j = 0; j < kLoads; ++j) {
                        uint32_t *word = reinterpret_cast<uint32_t *>(&vv[j]);
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c) {
                            const uint32_t is = __vcmpeq4(word[c] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                            if (is) {
#pragma unroll
                                for (uint32_t e = 0; e < 4; ++e)
                                    if (is >> (8 * e) & 1u) atomicMin(first_nan + piece * 16u + 4u * c + e, t0 + w * 32u + j * kPer + lane / kLanes);
                                *has_nan = 1;
                                word[c] &= ~is;
                            }
                        }
                    }
                }
                if (it > 1u) ok = __all_sync(0xFFFFFFFFu, bar_wait(v_free + 8 * stage, turn ^ 1u, abort_word));
                if (!ok) break;
                store(base + S::kV + stage * S::kTile, vv);
                bar_arrive(v_full + 8 * stage);
                id = id_next;
            }
            ++n_unit;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        // ---- softmax --------------------------------------------------------------------------------------------------------
        const uint32_t t = warp >> 2, l = tid & 127u, quarter = (warp & 3u) * 32u;
        const uint32_t s_mine = s_col[t] + (quarter << 16), o_mine = o_col[t] + (quarter << 16);
        for (uint32_t u = blockIdx.x; u < all && ok; u += gridDim.x) {
            const Unit x = unit_of(P, prefix, all - 1u - u);
            const uint32_t tiles = (x.most + kKeys - 1u) / kKeys;
            const uint32_t row = x.row0 + t * 128u + l, i_row = row / P.G, g = row % P.G;
            const bool real = row < x.n_rows, any_real = __any_sync(0xFFFFFFFFu, real);
            const uint32_t lim = real ? sees(P, x.r, i_row) : x.most;
            const uint32_t lim_least = __reduce_min_sync(0xFFFFFFFFu, lim);
            const int64_t head = int64_t(x.h * P.G + g);
            float m = -INFINITY, sum = 0.0f;
            if (tiles) {
                // the row as binary16, times a power of two that puts its largest magnitude in [2^13, 2^14) (see kv_cache.cu), with the sign of the scale
                uint4 w[D / 8];
                const T *src = static_cast<const T *>(P.x) + int64_t(x.r.row + i_row) * P.ldq + head * P.ldqh;
                float a = 0.0f;
#pragma unroll
                for (uint32_t c = 0; c < D / 8; ++c) {
                    w[c] = real ? __ldg(reinterpret_cast<const uint4 *>(src) + c) : make_uint4(0, 0, 0, 0);
                    a = fmaxf(a, fmaxf(fmaxf(fabsf(E::lo(w[c].x)), fabsf(E::hi(w[c].x))), fmaxf(fabsf(E::lo(w[c].y)), fabsf(E::hi(w[c].y)))));
                    a = fmaxf(a, fmaxf(fmaxf(fabsf(E::lo(w[c].z)), fabsf(E::hi(w[c].z))), fmaxf(fabsf(E::lo(w[c].w)), fabsf(E::hi(w[c].w)))));
                }
                const int32_t ea = int32_t(__float_as_uint(a) >> 23), up = ea == 0 || ea == 255 ? 0 : min(140 - ea, 100);
                const float mul = copysignf(pow2_biased(uint32_t(127 + up)), P.scale_log2), fac = fabsf(P.scale_log2) * pow2_biased(uint32_t(127 - up));
#pragma unroll
                for (uint32_t c = 0; c < D / 8; ++c) {
                    const uint32_t at = base + S::kQ + t * S::kTile + c / 8 * S::kHalf + l * 128u + (((c & 7u) ^ (l & 7u)) << 4);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(Fp16::two(E::lo(w[c].x) * mul, E::hi(w[c].x) * mul)), "r"(Fp16::two(E::lo(w[c].y) * mul, E::hi(w[c].y) * mul)),
                                 "r"(Fp16::two(E::lo(w[c].z) * mul, E::hi(w[c].z) * mul)), "r"(Fp16::two(E::lo(w[c].w) * mul, E::hi(w[c].w) * mul)) : "memory");
                }
                fence_proxy_async();
                bar_arrive(q_ready + 8 * t);
                for (uint32_t i = 0; i < tiles; ++i, ++it) {
                    ok = bar_wait(s_full + 8 * t, it & 1u, abort_word);
                    if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                    tc_after();
                    const uint32_t t0 = i * kKeys;
                    const float4 *meta = reinterpret_cast<const float4 *>(gen + S::kMeta) + (it & 3u) * 8u;
                    if (any_real) {
                        float low = 0.0f;
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k) low = fminf(low, meta[k].x);
                        auto tile = [&](auto edge_tag) {
                            constexpr bool kEdge = decltype(edge_tag)::value;
                            float top = -INFINITY;
#pragma unroll
                            for (uint32_t c = 0; c < 4; ++c) {
                                uint32_t v[32];
                                tc_load32(s_mine + 32 * c, v);
                                tc_loaded();
#pragma unroll
                                for (uint32_t k = 0; k < 2; ++k) {
                                    const float4 s = meta[2 * c + k];
                                    float best = -INFINITY;
#pragma unroll
                                    for (uint32_t e = 0; e < 16; ++e) {
                                        const float f = __uint_as_float(v[16 * k + e]);
                                        best = fmaxf(best, !kEdge || (t0 + 32 * c + 16 * k + e < lim && s.x >= 0.0f) ? f : -INFINITY);
                                    }
                                    const float here = fmaf(best, fac * s.x, s.y);
                                    top = fmaxf(top, kEdge && best == -INFINITY ? -INFINITY : here);
                                }
                            }
                            const bool move = top > m + kSlack;                          // (also from -infinity)
                            if (__any_sync(0xFFFFFFFFu, move)) {
                                const float f = move ? exp2_fast(m - top) : 1.0f;
                                if (move) m = top;
                                sum *= f;
                                if (i) {
#pragma unroll
                                    for (uint32_t c = 0; c < D / 32; ++c) {
                                        uint32_t v[32];
                                        tc_load32(o_mine + 32 * c, v);
                                        tc_loaded();
#pragma unroll
                                        for (uint32_t e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                                        tc_store32(o_mine + 32 * c, v);
                                    }
                                }
                            }
                            const float sub = m == -INFINITY ? 0.0f : m - kShift;
#pragma unroll
                            for (uint32_t c = 0; c < 4; ++c) {
                                uint32_t v[32], p[16];
                                tc_load32(s_mine + 32 * c, v);
                                tc_loaded();
#pragma unroll
                                for (uint32_t k = 0; k < 2; ++k) {
                                    const float4 s = meta[2 * c + k];
                                    const float by = fac * s.x, off = s.y - sub;
                                    float part = 0.0f;
#pragma unroll
                                    for (uint32_t e = 0; e < 16; e += 2) {
                                        float f[2];
#pragma unroll
                                        for (uint32_t z = 0; z < 2; ++z) {
                                            float d = fmaf(__uint_as_float(v[16 * k + e + z]), by, off);
                                            if (kEdge && (t0 + 32 * c + 16 * k + e + z >= lim || s.x < 0.0f)) d = -INFINITY;
                                            f[z] = exp2_fast(d);
                                            part += f[z];
                                        }
                                        p[8 * k + e / 2] = Fp16::two(f[0], f[1]);
                                    }
                                    sum += part * s.z;
                                }
                                tc_store16(s_mine + 16 * c, p);
                            }
                            tc_stored();
                        };
                        if (t0 + kKeys > lim_least || low < 0.0f) tile(std::true_type{});
                        else tile(std::false_type{});
                    }
                    tc_before();
                    bar_arrive(p_ready + 8 * t);
                }
                if (!ok) break;
                ok = bar_wait(o_full + 8 * t, n_unit & 1u, abort_word);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                tc_after();
            }
            // ---- the unit's rows --------------------------------------------------------------------------------------------
            const float inverse = sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
            T *dst = static_cast<T *>(P.o) + int64_t(x.r.row + i_row) * P.ldo + head * P.ldoh;
            const uint32_t *first_nan = nan_at + n_unit % kNanUnits * D;
            const bool has_nan = tiles && nan_at[kNanUnits * D + n_unit % kNanUnits] != 0;
            if (any_real) {
#pragma unroll
                for (uint32_t c = 0; c < D / 32; ++c) {
                    uint32_t v[32];
                    if (tiles) {
                        tc_load32(o_mine + 32 * c, v);
                        tc_loaded();
                    }
#pragma unroll
                    for (uint32_t e = 0; e < 32; ++e) {
                        float f = tiles && sum != 0.0f ? __uint_as_float(v[e]) * inverse : 0.0f;
                        if (has_nan && first_nan[32 * c + e] < lim) f = __uint_as_float(0x7FFFFFFFu);
                        v[e] = __float_as_uint(f);
                    }
                    if (real)
#pragma unroll
                        for (uint32_t e = 0; e < 32; e += 8)
                            *reinterpret_cast<uint4 *>(dst + 32 * c + e) =
                                make_uint4(E::two(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), E::two(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])),
                                           E::two(__uint_as_float(v[e + 4]), __uint_as_float(v[e + 5])), E::two(__uint_as_float(v[e + 6]), __uint_as_float(v[e + 7])));
                }
                if (real && P.lse) P.lse[int64_t(x.r.row + i_row) * P.Hq + head] = sum == 0.0f ? -INFINITY : (m - kShift + log2f(sum)) * 0.69314718055994531f;
            }
            tc_before();
            if (tiles) ++n_unit;
        }
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_prompts_status, 1u);
    if (warp == 12) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <class E, uint32_t D>
int launch(const AttendParams &P, cudaStream_t st) {
    static bool configured[64] = {};
    const int rc = op_configure(prompts_kernel<E, D>, PromptShape<D>::kSmem, configured);
    if (rc) return rc;
    return op_launch(prompts_kernel<E, D>, P.grid, kThreads, PromptShape<D>::kSmem, 1, st, P) == cudaSuccess ? EP_OK : EP_ERR_CUDA;
}

}  // namespace

// Units of 256 rows run one to an SM.  The other kernel takes 32 rows at a time, reads the cache again for each 32 and cuts along the tokens.
bool ep::prompts_serve(uint32_t N, uint32_t B, uint32_t G, uint32_t H) { return uint64_t(N) * G >= 128ull * B && uint64_t(N) * G * H >= 32ull * kUnitRows; }

int ep::launch_prompts(const AttendParams &P, uint32_t dim, int32_t dtype, cudaStream_t st) {
    if (dtype == EP_BF16) return dim == 64 ? launch<Bf16, 64>(P, st) : launch<Bf16, 128>(P, st);
    return dim == 64 ? launch<Fp16, 64>(P, st) : launch<Fp16, 128>(P, st);
}

int ep::op8_status_prompts() {
    unsigned int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_prompts_status, sizeof(v)) != cudaSuccess) return -1;
    if (v && cudaMemcpyToSymbol(g_prompts_status, &zero, sizeof(zero)) != cudaSuccess) return -1;
    return int(v);
}
