// Attention over the paged cache for many rows per request: prompts, and pieces of them.
#include "kv_cache.hpp"

using namespace ep;

namespace {

__device__ unsigned int g_prompts_status = 0;

// ======================================================================================================================
// A unit is 256 rows (a row = a query and one of the query heads that share a head of the cache) of one request and head, as two tiles
// of 128, against the request's tokens, 128 at a time.  For each 128 tokens the tensor cores need 2 * 2 * 256 * 128 * D operations in binary16, 2048
// cycles with D = 128, and the 256 * 128 exponentials at 16 per cycle and SM as many; a tile takes 4200.  What bounds it is the softmax
// of a row, one instruction after another: two warps to a scheduler, which spend half of their time at the exponentials and half at
// all that comes before and after (scores in, maximum, weights out), and registers leave no room for more warps.  Two prompts of up to
// 2048 rows x 40 heads on up to 4096 tokens 311 us, 838 TFLOP/s (calls of a graph; one after another from the host 337, 772).
//   warps 0 - 3, 4 - 7   a tile's softmax: a thread has a row.  Scores come from tensor memory, the weights go back there (binary16, over
//                        the scores) as the second product's left operand.
//   warps 8 - 11         bring keys and values in and turn them into binary16, exactly, in the layout of the products' right operands; the
//                        work for a token is shared by 256 rows.
//   warp 12              issues the products.  While one tile's softmax runs, the other's products do.
//   warp 13              the scales of the pages.  (On the way of the warps that bring the keys in, table, scale, logarithm one after
//                        the other, they took 700 cycles of every tile.)
// (Warps 14 and 15 have nothing to do: registers go from one group of four warps to another.)
// The running maximum is a reference m: it moves, and the accumulator in tensor memory is scaled, only when a score exceeds it by more
// than 2^8; weights are 2^(t - m + 7), so at most 2^15, inside binary16.  A page's value scale is taken into the exponent,
// t = score + log2(v_scale / one page's of the request), and out of the row's sum again.  (Weights made in one pass, in registers, with a check of their sums
// instead of the maximum first: 379 -> 462 us.  The two warps of a scheduler taking turns at the exponentials: 336 -> 360.  The next scores asked
// for before the weights are out: 311 -> 325.  A quarter of the exponentials as polynomials beside the unit: 311 -> 314, half: 335.)
// The loops are short on purpose: three roles run side by side, and what they execute over and over has to fit the SM's instruction
// cache (with everything unrolled, 170 KB, six of ten fetches hit it and a tile took 13 700 cycles).
// The tiles of tokens of all units form one list; every CTA takes an equal, contiguous share of it, as in kv_cache.cu, and what
// crosses a share goes through the workspace: units are few and long, and 640 of unequal length on 148 SMs left a third of them idle.
// ======================================================================================================================
constexpr uint32_t kUnitRows = 256, kKeys = 128, kHalfKeys = 64, kThreads = 32 * 16, kNanUnits = 8;
constexpr float kSlack = 8.0f, kShift = 7.0f;
// A piece of a unit in the workspace: O, four columns of all rows after another (a thread has a row, so a warp's store of four columns is 512
// bytes side by side), then m and l of each row.
template <uint32_t D>
constexpr uint32_t kPromptPiece = kUnitRows * (D + 2);

template <uint32_t D>
struct PromptShape {
    static constexpr uint32_t kHalves = D / 64, kHalf = 128 * 128, kTile = kHalves * kHalf;     // 128 rows x D binary16: blocks of 64 columns, 128-byte rows
    static constexpr uint32_t kQ = 0, kK = 2 * kTile, kV = kK + 2 * kTile;
    static constexpr uint32_t kMeta = kV + 2 * kTile;                  // four slots of eight groups of 16 tokens: key scale, log2 of the value scale's ratio, its inverse, the first value scale
    static constexpr uint32_t kNan = kMeta + 4 * 8 * 16;               // some units' first NaN token of each column, then their flags
    static constexpr uint32_t kBars = kNan + kNanUnits * (D + 1) * 4;
    static constexpr uint32_t kPart = kBars + 256, kPrefix = kPart + 128;      // (64 bytes for the sums' parts, then the share's first place)
    static constexpr uint32_t kSmem = kPrefix + 4 * (kMaxRequests + 32) + 1024;
    static_assert(kSmem <= 232448);
};

// the power of two that puts a row's largest magnitude in [2^13, 2^14); 0 for a row of zeros or with an infinity
__device__ __forceinline__ int32_t lifted(float largest) {
    const int32_t e = int32_t(__float_as_uint(largest) >> 23);
    return e == 0 || e == 255 ? 0 : min(140 - e, 100);
}
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}
// binary16 x binary16 to fp32, M = 128, N = n; `mn` = the right operand is MN-major
__host__ __device__ constexpr uint32_t f16_idesc(uint32_t n, uint32_t mn) { return (1u << 4) | (mn << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

__host__ __device__ __forceinline__ uint32_t sees(const AttendParams &P, const Extent &r, uint32_t query) {
    return !P.causal ? r.len : r.len + query + 1u > r.rows ? min(r.len, r.len + query + 1u - r.rows) : 0u;
}
// row tile j of a request: tokens that its last row sees; tiles of tokens, at least one, so that rows that see nothing are written too
__host__ __device__ __forceinline__ uint32_t most_of(const AttendParams &P, const Extent &r, uint32_t j) { return sees(P, r, (min((j + 1u) * kUnitRows, r.rows * P.G) - 1u) / P.G); }
__host__ __device__ __forceinline__ uint32_t tiles_of(const AttendParams &P, const Extent &r, uint32_t j) { return max(1u, (most_of(P, r, j) + kKeys - 1u) / kKeys); }
__host__ __device__ __forceinline__ uint32_t row_tiles_of(const AttendParams &P, const Extent &r) { return (r.rows * P.G + kUnitRows - 1u) / kUnitRows; }

// A unit's place in the list is its tiles and kStart before them, which is about what its start and end cost (rows in, the first
// tile and those at the diagonal the careful way, rows out).
constexpr uint32_t kStart = 3;
// a place in the list: requests, in them row tiles, in them heads, in them kStart and tiles of tokens
struct Place { uint32_t b, j, h, off, at, left; };        // at: number of place `off`; left: places of the share from there on

// What a CTA does next: tiles [first, first + count) of a unit.  Every role of the CTA walks its share alone.
struct Cursor {
    const AttendParams &P;
    Place p;
    Extent r;
    uint32_t total;               // tiles of the unit
    uint32_t first, count, taken; // taken: places of the share
    __host__ __device__ __forceinline__ Cursor(const AttendParams &P_, const Place &start) : P(P_), p(start) { enter(); }
    __host__ __device__ __forceinline__ void enter() {
        if (!p.left) return;
        for (;; ++p.b, p.j = 0) {                         // (p.left: there is one, unless somebody writes the lengths during the call: then a unit
            r = extent_of(P.q, p.b);                      // without rows at the last request, which the warp of the scales reports)
            if (p.j < row_tiles_of(P, r) || p.b + 1u >= P.q.B) break;
        }
        total = tiles_of(P, r, p.j);
        taken = P.workspace ? min(total + kStart - p.off, p.left) : total + kStart;
        first = max(p.off, kStart) - kStart;
        count = max(p.off + taken, kStart) - kStart - first;
    }
    __host__ __device__ __forceinline__ bool more() const { return p.left != 0; }
    __host__ __device__ __forceinline__ void next() {
        p.left -= min(p.left, taken);
        p.at += taken;
        p.off = 0;
        if (++p.h == P.q.H) p.h = 0, ++p.j;
        enter();
    }
    // tiles that take part in products (none where no row sees a token)
    __host__ __device__ __forceinline__ uint32_t products() const { return most_of(P, r, p.j) ? count : 0u; }
    __host__ __device__ __forceinline__ uint32_t row0() const { return p.j * kUnitRows; }
    // a unit of up to 128 rows has one tile of rows: nothing is done for the other
    __host__ __device__ __forceinline__ bool both() const { return row0() + kUnitRows / 2u < r.rows * P.G; }
    __host__ __device__ __forceinline__ uint32_t least() const { return sees(P, r, row0() / P.G); }
};

template <class E, uint32_t D>
__global__ void __launch_bounds__(kThreads, 1) prompts_kernel(const __grid_constant__ AttendParams P) {
    using S = PromptShape<D>;
    using T = typename E::T;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *gen = raw + (base - smem_u32(raw));
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    uint32_t *prefix = reinterpret_cast<uint32_t *>(gen + S::kPrefix), *nan_at = reinterpret_cast<uint32_t *>(gen + S::kNan);
    const uint32_t bars = base + S::kBars, k_full = bars, k_free = bars + 16, v_full = bars + 32, v_free = bars + 48, s_full = bars + 64, p_ready = bars + 96,
                   q_ready = bars + 128, o_full = bars + 144, o_moved = bars + 160, drained = bars + 176, rows_out = bars + 184, slot_addr = bars + 192,
                   abort_word = bars + 196;
    if (tid == 0) {
        for (uint32_t i = 0; i < 2; ++i) {
            bar_init(k_full + 8 * i, 129), bar_init(v_full + 8 * i, 128);
            bar_init(k_free + 8 * i, 1), bar_init(v_free + 8 * i, 1), bar_init(o_full + 8 * i, 1), bar_init(o_moved + 8 * i, 1);
            bar_init(q_ready + 8 * i, 128);
        }
        for (uint32_t i = 0; i < 4; ++i) bar_init(s_full + 8 * i, 1), bar_init(p_ready + 8 * i, 128);       // of tile t and buffer i: 2 t + i
        bar_init(drained, 1);
        bar_init(rows_out, 128);
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
    // places of a request: a warp adds up its row tiles; then sums over requests
    for (uint32_t b = warp; b < P.q.B; b += kThreads / 32u) {
        const Extent r = extent_of(P.q, b);
        uint32_t n = 0;
        for (uint32_t j = lane; j < row_tiles_of(P, r); j += 32u) n += tiles_of(P, r, j) + kStart;
        n = __reduce_add_sync(0xFFFFFFFFu, n);
        if (lane == 0) prefix[b] = n * P.q.H;
    }
    __syncthreads();
    const uint32_t all = prefix_sums(P.q.B, [&](uint32_t b) { return prefix[b]; }, P.most, prefix, reinterpret_cast<uint32_t *>(gen + S::kPart));
    if (all == 0 && blockIdx.x == 0 && tid == 0 && prefix[P.q.B]) atomicOr(&g_prompts_status, unsigned(kStatusPage));
    const uint32_t ctas = min(P.grid, all), u_begin = blockIdx.x < ctas ? uint32_t(uint64_t(all) * blockIdx.x / ctas) : 0u,
                   u_end = blockIdx.x < ctas ? uint32_t(uint64_t(all) * (blockIdx.x + 1u) / ctas) : 0u;
    Place *start = reinterpret_cast<Place *>(gen + S::kPart + 64);
    if (warp == 0) {
        Place p{0, 0, 0, 0, u_begin, u_end - u_begin};
        if (p.left) {
            p.b = request_of(prefix, 0, P.q.B, u_begin);
            const Extent r = extent_of(P.q, p.b);
            const uint32_t v = u_begin - prefix[p.b];
            uint32_t before = 0;                          // places of the row tiles before
            for (uint32_t j0 = 0;; j0 += 32u) {
                const uint32_t mine = j0 + lane < row_tiles_of(P, r) ? (tiles_of(P, r, j0 + lane) + kStart) * P.q.H : 0u;
                uint32_t inc = mine;
#pragma unroll
                for (uint32_t d = 1; d < 32; d <<= 1) {
                    const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                    if (lane >= d) inc += o;
                }
                const uint32_t here = __ballot_sync(0xFFFFFFFFu, mine && before + inc > v);
                if (here) {
                    const uint32_t k = __ffs(int(here)) - 1u, per_head = __shfl_sync(0xFFFFFFFFu, mine, k) / P.q.H, from = before + __shfl_sync(0xFFFFFFFFu, inc - mine, k);
                    p.j = j0 + k, p.h = (v - from) / per_head, p.off = (v - from) % per_head;
                    if (!P.workspace && p.off) {          // units are not cut: the next one that begins in this share
                        const uint32_t skip = per_head - p.off;
                        p.left -= min(p.left, skip);
                        p.at += skip, p.off = 0;
                        if (++p.h == P.q.H) p.h = 0, ++p.j;
                    }
                    break;
                }
                before += __shfl_sync(0xFFFFFFFFu, inc, 31);
                if (j0 >= row_tiles_of(P, r)) {           // (see Cursor::enter)
                    p.left = 0;
                    if (lane == 0) atomicOr(&g_prompts_status, unsigned(kStatusPage));
                    break;
                }
            }
        }
        if (lane == 0) *start = p;
    }
    __syncthreads();
    const Place begin = *start;
    uint32_t *desc = P.workspace ? reinterpret_cast<uint32_t *>(P.workspace) + blockIdx.x * 8u : nullptr;
    if (desc && tid == 0) desc[3] = 0;
    __syncthreads();
    // tensor memory: two buffers of scores (and weights) of each tile, 64 columns each, then the accumulators
    const uint32_t o_col[2] = {tmem + 256u, tmem + 384u};
    uint32_t it = 0, n_unit = 0;                          // tiles of tokens and units so far
    bool ok = true;

    // registers: 512 threads x 128 at launch = 128 x (168 + 168 + 104 + 72)
    if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ---- products -----------------------------------------------------------------------------------------------------
        if (warp == 12) {
            const uint32_t lead = elected();
            constexpr uint32_t kScores = f16_idesc(kHalfKeys, 0), kValues = f16_idesc(D, 1);
            // half n of a unit's tokens: 64 of them, buffer n mod 2; `stage`: where its 128 tokens lie
            auto scores = [&](uint32_t t, uint32_t n, uint32_t stage) {
                // (descriptors differ in their address, 16 bytes a step of it: 32 bytes further along the swizzled rows, then the next 64 columns)
                const uint64_t a = operand_desc(base + S::kQ + t * S::kTile), b = operand_desc(base + S::kK + stage * S::kTile + (n & 1u) * kHalfKeys * 128u);
#pragma unroll
                for (uint32_t k = 0; k < D / 16; ++k) {
                    const uint32_t at = (k / 4 * S::kHalf + k % 4 * 32) >> 4;
                    mma_f16_ss(tmem + t * 128u + (n & 1u) * 64u, a + at, b + at, kScores, k ? 1u : 0u, lead);
                }
                tc_commit(s_full + 8 * (2 * t + (n & 1u)), lead);
            };
            auto values = [&](uint32_t t, uint32_t n, uint32_t stage) {
                const uint64_t b = operand_desc(base + S::kV + stage * S::kTile + (n & 1u) * kHalfKeys * 128u, S::kHalf);
#pragma unroll
                for (uint32_t k = 0; k < kHalfKeys / 16; ++k)
                    mma_f16_ts(t ? o_col[1] : o_col[0], tmem + t * 128u + (n & 1u) * 64u + 8 * k, b + k * (2048 >> 4), kValues, n | k ? 1u : 0u, lead);
                tc_commit(o_moved + 8 * t, lead);
            };
            // Scores run two halves ahead of the weights, so that a tile's softmax finds its next scores ready.  (Scores of 128 tokens at
            // a time in one buffer: softmax, second product, first product one after the other for each tile of rows, 340 us.)
            uint32_t it1 = 0, n_unit1 = 0;                // of the second tile of rows
            for (Cursor x(P, begin); x.more() && ok; x.next()) {
                const uint32_t tiles = x.products(), halves = 2u * tiles;
                const bool both = x.both();
                if (tiles == 0) continue;
                // Units of one tile of rows: the second tile's warps take no part in them, and must have done with the unit before (its
                // record of NaN is cleared some units later).
                if (!both && n_unit1) ok = bar_wait_warp(rows_out, (n_unit1 - 1u) & 1u, abort_word);
                ok = ok && bar_wait_warp(k_full + 8 * (it & 1u), (it >> 1) & 1u, abort_word) && bar_wait_warp(q_ready, n_unit & 1u, abort_word);
                if (!ok) break;
                tc_after();
                scores(0, 0, it & 1u);
                if (both) {
                    ok = bar_wait_warp(q_ready + 8, n_unit1 & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    scores(1, 0, it & 1u);
                }
                scores(0, 1, it & 1u);
                if (both) scores(1, 1, it & 1u);
                tc_commit(k_free + 8 * (it & 1u), lead);
#pragma unroll 1
                for (uint32_t n = 0; n < halves; ++n) {
                    const uint32_t now = it + n / 2u, stage = now & 1u, later = now + 1u, ahead = later & 1u;
                    const bool more = n + 2u < halves;
                    if (!(n & 1u)) ok = bar_wait_warp(v_full + 8 * stage, (now >> 1) & 1u, abort_word);
                    ok = ok && bar_wait_warp(p_ready + 8 * (n & 1u), now & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    values(0, n, stage);
                    if (more) {
                        if (!(n & 1u)) ok = bar_wait_warp(k_full + 8 * ahead, (later >> 1) & 1u, abort_word);
                        if (!ok) break;
                        tc_after();
                        scores(0, n + 2u, ahead);
                    }
                    if (both) {
                        ok = bar_wait_warp(p_ready + 8 * (2u + (n & 1u)), (it1 + n / 2u) & 1u, abort_word);
                        if (!ok) break;
                        tc_after();
                        values(1, n, stage);
                        if (more) scores(1, n + 2u, ahead);
                    }
                    if (n & 1u) {
                        tc_commit(v_free + 8 * stage, lead);
                        if (more) tc_commit(k_free + 8 * ahead, lead);
                    }
                }
                if (!ok) break;
                tc_commit(o_full, lead);
                if (both) {
                    tc_commit(o_full + 8, lead);
                    ++n_unit1;
                    it1 += tiles;
                }
                it += tiles;
                ++n_unit;
            }
            tc_commit(drained, lead);
            bar_drain(drained, 0);                        // nothing is in flight when tensor memory is given back
        }
        if (warp == 13) {
            // ---- scales ---------------------------------------------------------------------------------------------------
            // of groups of 16 tokens, lane = group: the page of tile i + 2 and the scales of tile i + 1 are on their way while tile i's are written
            for (Cursor x(P, begin); x.more() && ok; x.next()) {
                const uint32_t tiles = x.products(), t_first = x.first * kKeys;
                if (lane == 0 && x.row0() >= x.r.rows * P.G) atomicOr(&g_prompts_status, unsigned(kStatusPage));       // (see Cursor::enter)
                if (tiles == 0) continue;
                const int32_t *table = P.q.table + int64_t(x.p.b) * P.q.ldt;
                const float vs_first = first_scale(P.q, P.vs, x.p.b, x.p.h, x.r.len), per_first = __frcp_rn(vs_first);
                auto page_at = [&](uint32_t i) {          // -1: no token, or (reported by the warps that bring it in) no page
                    const uint32_t t = t_first + i * kKeys + 16u * lane;
                    const int32_t id = lane < 8 && i < tiles && t < x.r.len ? __ldg(table + (t >> P.q.shift)) : -1;
                    return uint32_t(id) < P.q.pages ? id : -1;
                };
                auto scales_at = [&](int32_t page, float &ks, float &vs) {
                    const size_t block = size_t(uint32_t(max(page, 0))) * P.q.H + x.p.h;
                    ks = page >= 0 ? __ldg(P.ks + block) : -1.0f;
                    vs = page >= 0 ? __ldg(P.vs + block) : 1.0f;
                };
                float ks, vs, ks_next, vs_next;
                scales_at(page_at(0), ks, vs);
                int32_t page = page_at(1);
#pragma unroll 1
                for (uint32_t i = 0; i < tiles; ++i, ++it) {
                    scales_at(page, ks_next, vs_next);
                    page = page_at(i + 2u);
                    const uint32_t stage = it & 1u;
                    if (it > 1u) ok = bar_wait_warp(k_free + 8 * stage, (it >> 1 & 1u) ^ 1u, abort_word);
                    if (!ok) break;
                    const float some = fmaxf(vs * per_first, kLeastRatio);
                    if (lane < 8) *reinterpret_cast<float4 *>(gen + S::kMeta + ((it & 3u) * 8u + lane) * 16u) = make_float4(ks, log2f(some), __fdiv_rn(1.0f, some), vs_first);
                    __syncwarp();
                    if (lane == 0) bar_arrive(k_full + 8 * stage);
                    ks = ks_next, vs = vs_next;
                }
            }
        }
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        // ---- keys and values ----------------------------------------------------------------------------------------------
        constexpr uint32_t kLanes = D / 16, kPer = 32 / kLanes, kLoads = 32 / kPer;          // lanes of a token; tokens of a load; loads of a warp's 32 tokens
        const uint32_t w = warp - 8u, l = tid - 256u, piece = lane % kLanes, half = piece >> 2;
        // where a lane's first piece goes, of even and odd loads: its row's number mod 8 swizzles the 16-byte pieces
        uint32_t to[2];
#pragma unroll
        for (uint32_t odd = 0; odd < 2; ++odd) {
            const uint32_t row = w * 32u + lane / kLanes, sw = (row + odd * 4u) & 7u;
            to[odd] = half * S::kHalf + row * 128u + (((2u * (piece & 3u) + (half ? 1u : 0u)) ^ sw) << 4);
        }
        for (Cursor x(P, begin); x.more() && ok; x.next()) {
            const uint32_t tiles = x.products(), t_first = x.first * kKeys, least = x.least();
            if (tiles == 0) continue;
            const int32_t *table = P.q.table + int64_t(x.p.b) * P.q.ldt;
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
                atomicOr(&g_prompts_status, unsigned(kStatusPage));
                return -1;
            };
            // a warp's 32 tokens lie in one page or two, 16 in each
            auto load = [&](const uint8_t *cache, uint32_t t0, int32_t id0, int32_t id1, uint4 (&v)[kLoads]) {
#pragma unroll
                for (uint32_t side = 0; side < 2; ++side) {
                    const int32_t page = side ? id1 : id0;
                    const uint8_t *src = cache + (((uint64_t(uint32_t(page)) * P.q.H + x.p.h) << P.q.shift) + ((t0 + w * 32u + side * 16u) & (P.q.page - 1u)) + lane / kLanes) * D + piece * 16u;
#pragma unroll
                    for (uint32_t j = side * kLoads / 2; j < (side + 1) * kLoads / 2; ++j) {
                        v[j] = make_uint4(0, 0, 0, 0);
                        if (page >= 0)
                            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(v[j].x), "=r"(v[j].y), "=r"(v[j].z), "=r"(v[j].w) : "l"(src + (j - side * kLoads / 2) * kPer * D));
                    }
                }
            };
            // 16 values of a token: two 16-byte pieces of its row in the block of 64 columns; the two halves of a row write
            // them in opposite order, to different banks
            auto store = [&](uint32_t at, const uint4 (&v)[kLoads]) {
#pragma unroll
                for (uint32_t j = 0; j < kLoads; ++j) {
                    const bool flip = half != 0;
                    uint32_t f[8];
                    f16x4_of_e4m3x4(flip ? v[j].z : v[j].x, f[0], f[1]);
                    f16x4_of_e4m3x4(flip ? v[j].w : v[j].y, f[2], f[3]);
                    f16x4_of_e4m3x4(flip ? v[j].x : v[j].z, f[4], f[5]);
                    f16x4_of_e4m3x4(flip ? v[j].y : v[j].w, f[6], f[7]);
                    const uint32_t a0 = at + to[kPer == 4 ? j & 1u : 0u] + j * kPer * 128u;
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a0), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a0 ^ 16u), "r"(f[4]), "r"(f[5]), "r"(f[6]), "r"(f[7]) : "memory");
                }
            };
            // Values of a tile that some rows do not see all of: tokens past the request's end may hold anything and become zeros, and a
            // NaN counts for the rows that see its token only - it is taken out here and put into those rows at the unit's end.
            auto scrub = [&](uint32_t at, uint32_t t0) {
#pragma unroll 1
                for (uint32_t j = 0; j < 2 * kLoads; ++j) {
                    const uint32_t load_no = j >> 1, token = t0 + w * 32u + load_no * kPer + lane / kLanes;
                    const uint32_t a0 = (at + (kPer == 4 && load_no & 1u ? to[1] : to[0]) + load_no * kPer * 128u) ^ (j & 1u ? 16u : 0u);
                    const uint4 v = ld_smem16(a0);
                    if (token >= x.r.len) {
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(a0), "r"(0u) : "memory");
                    } else {
                        const uint32_t word[4] = {v.x, v.y, v.z, v.w};
                        const uint32_t first = piece * 16u + ((j & 1u) != half ? 8u : 0u);           // (see store: which eight of the sixteen)
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c)
                            if ((word[c] & 0x7FFFu) > 0x7C00u || (word[c] & 0x7FFF0000u) > 0x7C000000u) {
                                *has_nan = 1;
                                if ((word[c] & 0x7FFFu) > 0x7C00u) atomicMin(first_nan + first + 2u * c, token);
                                if ((word[c] & 0x7FFF0000u) > 0x7C000000u) atomicMin(first_nan + first + 2u * c + 1u, token);
                                st_smem(a0 + 4u * c, ((word[c] & 0x7FFFu) > 0x7C00u ? 0u : word[c] & 0xFFFFu) | ((word[c] & 0x7FFF0000u) > 0x7C000000u ? 0u : word[c] & 0xFFFF0000u));
                            }
                    }
                }
            };
            uint4 kv[kLoads], vv[kLoads];
            int32_t id0 = page_at(t_first + w * 32u), id1 = page_at(t_first + w * 32u + 16u);
            load(P.k, t_first, id0, id1, kv);
            load(P.v, t_first, id0, id1, vv);
            if (tiles > 1) id0 = page_at(t_first + kKeys + w * 32u), id1 = page_at(t_first + kKeys + w * 32u + 16u);
#pragma unroll 1
            for (uint32_t i = 0; i < tiles; ++i, ++it) {
                const uint32_t stage = it & 1u, turn = (it >> 1) & 1u, t0 = t_first + i * kKeys;
                if (it > 1u) ok = __all_sync(0xFFFFFFFFu, bar_wait(k_free + 8 * stage, turn ^ 1u, abort_word));
                if (!ok) break;
                store(base + S::kK + stage * S::kTile, kv);
                fence_proxy_async();
                bar_arrive(k_full + 8 * stage);
                if (i + 1u < tiles) {
                    load(P.k, t0 + kKeys, id0, id1, kv);
                }
                if (it > 1u) ok = __all_sync(0xFFFFFFFFu, bar_wait(v_free + 8 * stage, turn ^ 1u, abort_word));
                if (!ok) break;
                store(base + S::kV + stage * S::kTile, vv);
                if (t0 + kKeys > least) scrub(base + S::kV + stage * S::kTile, t0);
                fence_proxy_async();
                bar_arrive(v_full + 8 * stage);
                if (i + 1u < tiles) {
                    load(P.v, t0 + kKeys, id0, id1, vv);
                    if (i + 2u < tiles) id0 = page_at(t0 + 2 * kKeys + w * 32u), id1 = page_at(t0 + 2 * kKeys + w * 32u + 16u);
                }
            }
            ++n_unit;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        // ---- softmax --------------------------------------------------------------------------------------------------------
        const uint32_t t = warp >> 2, l = tid & 127u, quarter = (warp & 3u) * 32u;
        const uint32_t s_mine = tmem + t * 128u + (quarter << 16), o_mine = (t ? o_col[1] : o_col[0]) + (quarter << 16);
        // Rows of a unit's tile as binary16, times a power of two that puts a row's largest magnitude in [2^13, 2^14) (see kv_cache.cu),
        // with the sign of the scale; returns the factor of the row's scores.  They go in as soon as the scores of the unit before are done.
        auto rows_in = [&](const Cursor &y) {
            // A warp's 32 rows, 16 bytes to a lane: D / 8 lanes side by side have a row (a row to a lane: 32 places 256 bytes apart in every load).
            // In loops, by way of shared memory: the first unit's rows come while nothing of this code is in the instruction cache.
            constexpr uint32_t kLanes = D / 8, kPer = 32 / kLanes;
            const uint32_t row = y.row0() + t * 128u + l, i_row = row / P.G, n_rows = y.r.rows * P.G, sub = lane / kLanes, c = lane % kLanes;
            const T *src = static_cast<const T *>(P.x) + int64_t(y.r.row + i_row) * P.ldq + int64_t(y.p.h * P.G + row % P.G) * P.ldqh;
            auto place = [&](uint32_t k) {
                const uint32_t in_tile = (warp & 3u) * 32u + k * kPer + sub;
                return base + S::kQ + t * S::kTile + c / 8 * S::kHalf + in_tile * 128u + (((c & 7u) ^ (in_tile & 7u)) << 4);
            };
#pragma unroll 4
            for (uint32_t k = 0; k < kLanes; ++k) {
                const T *from = reinterpret_cast<const T *>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(src), k * kPer + sub));
                const bool there = row - lane + k * kPer + sub < n_rows;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(place(k)), "l"(there ? from + c * 8u : static_cast<const T *>(P.x)), "r"(there ? 16u : 0u) : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            float largest = 0.0f;                         // of this lane's row
#pragma unroll 1
            for (uint32_t k0 = 0; k0 < kLanes; k0 += 4) { // (what this lane has brought, four rows' chains side by side)
                uint4 w[4];
                float a[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) w[k] = ld_smem16(place(k0 + k));
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    a[k] = max3(max3(fabsf(E::lo(w[k].x)), fabsf(E::hi(w[k].x)), fabsf(E::lo(w[k].y))), fabsf(E::hi(w[k].y)), fabsf(E::lo(w[k].z)));
                    a[k] = max3(a[k], max3(fabsf(E::hi(w[k].z)), fabsf(E::lo(w[k].w)), fabsf(E::hi(w[k].w))), 0.0f);
                }
#pragma unroll
                for (uint32_t x = 1; x < kLanes; x <<= 1)
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) a[k] = fmaxf(a[k], __shfl_xor_sync(0xFFFFFFFFu, a[k], x));
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const float mine = __shfl_sync(0xFFFFFFFFu, a[k], lane % kPer * kLanes);
                    if (lane / kPer == k0 + k) largest = mine;
                }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const float mul = copysignf(pow2_biased(uint32_t(127 + lifted(a[k]))), P.scale_log2);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(place(k0 + k)), "r"(Fp16::two(E::lo(w[k].x) * mul, E::hi(w[k].x) * mul)), "r"(Fp16::two(E::lo(w[k].y) * mul, E::hi(w[k].y) * mul)),
                                 "r"(Fp16::two(E::lo(w[k].z) * mul, E::hi(w[k].z) * mul)), "r"(Fp16::two(E::lo(w[k].w) * mul, E::hi(w[k].w) * mul)) : "memory");
                }
            }
            fence_proxy_async();
            bar_arrive(q_ready + 8 * t);
            return fabsf(P.scale_log2) * pow2_biased(uint32_t(127 - lifted(largest)));
        };
        float fac_next = 0.0f;
        bool rows_there = false;                          // of the unit that comes
        uint32_t done = 0, n_done = 0;                    // tiles and units that this tile of rows took part in (it, n_unit: all)
        Cursor y(P, begin);                               // the unit after x
#pragma unroll 1
        for (Cursor x(P, begin); x.more() && ok; x.next()) {
            y.next();
            const uint32_t tiles = x.products(), n_rows = x.r.rows * P.G;
            if (t && !x.both()) {
                it += tiles;
                if (tiles) ++n_unit;
                continue;
            }
            const uint32_t row = x.row0() + t * 128u + l, i_row = row / P.G, g = row % P.G;
            const bool real = row < n_rows, any_real = __any_sync(0xFFFFFFFFu, real);
            const uint32_t lim = real ? sees(P, x.r, i_row) : most_of(P, x.r, x.p.j);
            const uint32_t lim_least = __reduce_min_sync(0xFFFFFFFFu, lim);
            const int64_t head = int64_t(x.p.h * P.G + g);
            float m = -INFINITY, sum = 0.0f, vs_first = 1.0f;
            if (tiles) {
                if (!rows_there) fac_next = rows_in(x);
                const float fac = fac_next;
                rows_there = false;
#pragma unroll 1
                for (uint32_t n = 0; n < 2u * tiles; ++n) {
                    const uint32_t buffer = n & 1u, turn = done + n / 2u;
                    ok = bar_wait_warp(s_full + 8 * (2 * t + buffer), turn & 1u, abort_word);
                    if (!ok) break;
                    tc_after();
                    const uint32_t t0 = x.first * kKeys + n * kHalfKeys, s_at = s_mine + buffer * 64u;
                    const float4 *meta = reinterpret_cast<const float4 *>(gen + S::kMeta) + ((it + n / 2u) & 3u) * 8u + buffer * 4u;
                    if (any_real) {
                        float4 scale[4];
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) scale[k] = meta[k];
                        vs_first = scale[0].w;
                        const bool out = fminf(fminf(scale[0].x, scale[1].x), fminf(scale[2].x, scale[3].x)) < 0.0f;
                        auto tile = [&](auto edge_tag) {
                            constexpr bool kEdge = decltype(edge_tag)::value;
                            uint32_t v[2][32];
                            tc_load32(s_at, v[0]);
                            tc_load32(s_at + 32, v[1]);
                            tc_loaded32(v[0]);
                            tc_loaded32(v[1]);
                            float top = -INFINITY;
#pragma unroll
                            for (uint32_t k = 0; k < 4; ++k) {
                                float best = -INFINITY;
#pragma unroll
                                for (uint32_t e = 0; e < 16; e += 2) {
                                    float f[2];
#pragma unroll
                                    for (uint32_t z = 0; z < 2; ++z) {
                                        uint32_t &w = v[k / 2][16 * (k % 2) + e + z];
                                        if (kEdge && (t0 + 16 * k + e + z >= lim || scale[k].x < 0.0f)) w = 0xFF800000u;        // -infinity
                                        f[z] = __uint_as_float(w);
                                    }
                                    best = max3(best, f[0], f[1]);
                                }
                                const float here = fmaf(best, fac * scale[k].x, scale[k].y);
                                top = fmaxf(top, kEdge && best == -INFINITY ? -INFINITY : here);
                            }
                            const bool move = top > m + kSlack;                          // (also from -infinity)
                            if (__any_sync(0xFFFFFFFFu, move)) {
                                const float f = move ? exp2_fast(m - top) : 1.0f;
                                if (move) m = top;
                                sum *= f;
                                if (n) {
                                    ok = bar_wait_warp(o_moved + 8 * t, (2u * done + n - 1u) & 1u, abort_word);       // (the half before is in the accumulator)
                                    tc_after();
#pragma unroll 1
                                    for (uint32_t c = 0; c < D; c += 16) {
                                        uint32_t a[16];
                                        tc_load16(o_mine + c, a);
                                        tc_loaded16(a);
#pragma unroll
                                        for (uint32_t e = 0; e < 16; ++e) a[e] = __float_as_uint(__uint_as_float(a[e]) * f);
                                        tc_store16(o_mine + c, a);
                                    }
                                }
                            }
                            const float sub = m == -INFINITY ? 0.0f : m - kShift;
                            uint32_t p[32];
#pragma unroll
                            for (uint32_t k = 0; k < 4; ++k) {
                                const float by = fac * scale[k].x, off = scale[k].y - sub;
                                const uint64_t by2 = pair_of(by, by), off2 = pair_of(off, off);
                                uint64_t part = 0;
#pragma unroll
                                for (uint32_t e = 0; e < 16; e += 2) {
                                    const uint32_t w0 = v[k / 2][16 * (k % 2) + e], w1 = v[k / 2][16 * (k % 2) + e + 1];
                                    float f[2];
                                    pair_to(fma2(pair_of(__uint_as_float(w0), __uint_as_float(w1)), by2, off2), f[0], f[1]);
                                    if (kEdge) f[0] = w0 == 0xFF800000u ? -INFINITY : f[0], f[1] = w1 == 0xFF800000u ? -INFINITY : f[1];       // (by may be 0 or negative)
                                    f[0] = exp2_fast(f[0]), f[1] = exp2_fast(f[1]);
                                    part = add2(part, pair_of(f[0], f[1]));
                                    p[8 * k + e / 2] = Fp16::two(f[0], f[1]);
                                }
                                float odd, even;
                                pair_to(part, even, odd);
                                sum = fmaf(even + odd, scale[k].z, sum);
                            }
                            tc_store32(s_at, p);                                         // over the scores, which have been read
                            tc_stored();
                        };
                        if (t0 + kHalfKeys > lim_least || out) tile(std::true_type{});
                        else tile(std::false_type{});
                    }
                    tc_before();
                    bar_arrive(p_ready + 8 * (2 * t + buffer));
                }
                it += tiles;
                done += tiles;
                if (!ok) break;
                if (y.more() && y.products() && (!t || y.both())) {
                    fac_next = rows_in(y);
                    rows_there = true;
                }
                ok = bar_wait(o_full + 8 * t, n_done & 1u, abort_word);
                if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                tc_after();
            }
            // ---- the unit's rows, or a piece of them --------------------------------------------------------------------------
            if (x.count == 0) continue;                   // (a share that ends before the unit's first tile)
            const bool whole = x.count == x.total;
            const float inverse = sum == 0.0f ? 0.0f : whole ? __fdiv_rn(vs_first, sum) : vs_first;
            T *dst = static_cast<T *>(P.o) + int64_t(x.r.row + i_row) * P.ldo + head * P.ldoh;
            float *piece = whole ? nullptr : P.workspace + size_t(P.grid) * 8u + (size_t(blockIdx.x) * 2u + (x.first ? 0u : 1u)) * kPromptPiece<D>;
            const uint32_t *first_nan = nan_at + n_unit % kNanUnits * D;
            const bool has_nan = tiles && nan_at[kNanUnits * D + n_unit % kNanUnits] != 0;
            if (any_real) {
#pragma unroll 1
                for (uint32_t c = 0; c < D / 32; ++c) {
                    uint32_t v[32];
                    if (tiles) {
                        tc_load32(o_mine + 32 * c, v);
                        tc_loaded32(v);
                    }
#pragma unroll
                    for (uint32_t e = 0; e < 32; ++e) {
                        float f = tiles && sum != 0.0f ? __uint_as_float(v[e]) * inverse : 0.0f;
                        if (has_nan && first_nan[32 * c + e] < lim) f = __uint_as_float(0x7FFFFFFFu);
                        v[e] = __float_as_uint(f);
                    }
                    if (!whole) {
#pragma unroll
                        for (uint32_t e = 0; e < 32; e += 4)
                            *reinterpret_cast<uint4 *>(piece + ((8 * c + e / 4) * kUnitRows + t * 128u + l) * 4u) = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    } else {
                        // 32 columns of the warp's rows, turned in shared memory so that four lanes write a row's 64 bytes
                        const uint32_t mine = base + S::kPrefix + warp * 2048u;
#pragma unroll
                        for (uint32_t e = 0; e < 32; e += 8)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(mine + lane * 64u + ((e / 8 ^ (lane >> 1 & 3u)) << 4)), "r"(E::two(__uint_as_float(v[e]), __uint_as_float(v[e + 1]))),
                                         "r"(E::two(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]))), "r"(E::two(__uint_as_float(v[e + 4]), __uint_as_float(v[e + 5]))),
                                         "r"(E::two(__uint_as_float(v[e + 6]), __uint_as_float(v[e + 7]))) : "memory");
                        __syncwarp();
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) {
                            const uint32_t other = 8 * k + (lane >> 2);
                            T *to = reinterpret_cast<T *>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(dst), other));
                            const uint4 w = ld_smem16(mine + other * 64u + (((lane & 3u) ^ (other >> 1 & 3u)) << 4));
                            if (row - lane + other < n_rows) *reinterpret_cast<uint4 *>(to + 32 * c + 8 * (lane & 3u)) = w;
                        }
                        __syncwarp();
                    }
                }
                if (!whole) {
                    piece[kUnitRows * D + t * 128u + l] = m;
                    piece[kUnitRows * (D + 1) + t * 128u + l] = sum;
                } else if (real && P.lse) {
                    P.lse[int64_t(x.r.row + i_row) * P.Hq + head] = sum == 0.0f ? -INFINITY : (m - kShift + log2f(sum)) * 0.69314718055994531f;
                }
            }
            if (!whole && x.first == 0 && tid == 0) {     // this CTA begins the unit: the second launch joins it from here
                const uint32_t end = x.p.at - x.p.off + x.total + kStart;
                uint32_t cta = uint32_t(uint64_t(end - 1u) * ctas / all);
                while (uint64_t(all) * (cta + 1u) / ctas < end) ++cta;
                while (uint64_t(all) * cta / ctas >= end) --cta;
                desc[0] = x.p.b, desc[1] = x.p.j, desc[2] = x.p.h, desc[3] = cta + 1u;
            }
            tc_before();
            if (tiles) {
                ++n_unit, ++n_done;
                if (t) bar_arrive(rows_out);
            }
        }
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && ld_smem(abort_word)) atomicOr(&g_prompts_status, unsigned(kStatusWait));
    if (warp == 12) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// The units that cross a share: CTA column k takes the one that CTA k of the first launch began; its other pieces are those of the CTAs
// after it, in order (a CTA's first piece continues a unit, its second begins one).  A thread has four columns of a row.
template <class E, uint32_t D>
__global__ void __launch_bounds__(256) prompts_join_kernel(const __grid_constant__ AttendParams P) {
    using T = typename E::T;
    op_wait_for_stream();
    const uint32_t *desc = reinterpret_cast<const uint32_t *>(P.workspace) + blockIdx.x * 8u;
    const uint32_t end = desc[3];
    if (end == 0) return;
    const uint32_t b = desc[0], j = desc[1], h = desc[2], n = end - blockIdx.x - 1u;
    const Extent r = extent_of(P.q, b);
    const float *pieces = P.workspace + size_t(P.grid) * 8u;
    const float *own = pieces + (size_t(blockIdx.x) * 2u + 1u) * kPromptPiece<D>, *first = pieces + size_t(blockIdx.x + 1u) * 2u * kPromptPiece<D>;
    // eight lanes have eight rows of the same columns, as they lie in the pieces; four such groups write 32 bytes of each row
    const uint32_t group = threadIdx.x >> 3, d = group % (D / 4u) * 4u, row = blockIdx.y * (1024u / D) + group / (D / 4u) * 8u + (threadIdx.x & 7u), place = (d * kUnitRows) + row * 4u;
    const uint32_t at = j * kUnitRows + row, i = at / P.G, g = at % P.G;
    if (at >= r.rows * P.G) return;
    const float own_top = own[kUnitRows * D + row];
    float top = own_top;
#pragma unroll 4
    for (uint32_t c = 0; c < n; ++c) top = fmaxf(top, first[size_t(c) * 2u * kPromptPiece<D> + kUnitRows * D + row]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float f = exp2_fast(own_top - ref), sum = own[kUnitRows * (D + 1) + row] * f;
    float4 acc = *reinterpret_cast<const float4 *>(own + place);
    acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
#pragma unroll 4
    for (uint32_t c = 0; c < n; ++c) {
        const float *p = first + size_t(c) * 2u * kPromptPiece<D>;
        f = exp2_fast(p[kUnitRows * D + row] - ref);
        sum += p[kUnitRows * (D + 1) + row] * f;
        const float4 v = *reinterpret_cast<const float4 *>(p + place);
        acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
    }
    const float inverse = sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
    const int64_t t = int64_t(r.row + i), head = int64_t(h * P.G + g);
    *reinterpret_cast<uint2 *>(static_cast<T *>(P.o) + t * P.ldo + head * P.ldoh + d) = make_uint2(E::two(acc.x * inverse, acc.y * inverse), E::two(acc.z * inverse, acc.w * inverse));
    if (P.lse && d == 0) P.lse[t * P.Hq + head] = sum == 0.0f ? -INFINITY : (top - kShift + log2f(sum)) * 0.69314718055994531f;
}

template <class E, uint32_t D>
int launch(const AttendParams &P, cudaStream_t st) {
    static bool configured[64] = {};
    const int rc = op_configure(prompts_kernel<E, D>, PromptShape<D>::kSmem, configured);
    if (rc) return rc;
    if (op_launch(prompts_kernel<E, D>, P.grid, kThreads, PromptShape<D>::kSmem, 1, st, P) != cudaSuccess) return EP_ERR_CUDA;
    if (P.workspace && op_launch(prompts_join_kernel<E, D>, dim3(P.grid, kUnitRows * D / 4u / 256u), 256, 0, 1, st, P) != cudaSuccess) return EP_ERR_CUDA;
    return EP_OK;
}

const bool registered = ep::add_status_word([] { return op_status(g_prompts_status); });

}  // namespace

// Rows enough to fill part of the products' 256: the other kernel takes 8 or 16 at a time and reads the cache again for each such tile (16 requests of
// 4 rows x 8 heads on 8192 tokens: 124 us there, 97 here).
bool ep::prompts_serve(uint32_t N, uint32_t B, uint32_t G) { return uint64_t(N) * G > 16ull * B; }

size_t ep::prompts_workspace_bytes(uint32_t grid, uint32_t dim) { return size_t(grid) * (8u + 2u * kUnitRows * (size_t(dim) + 2u)) * 4u; }

int ep::launch_prompts(AttendParams P, size_t workspace_bytes, bool cut, uint32_t dim, int32_t dtype, cudaStream_t st) {
    if (!cut) P.workspace = nullptr;
    else if (!P.workspace || workspace_bytes < prompts_workspace_bytes(P.grid, dim) || (reinterpret_cast<uintptr_t>(P.workspace) & 15u)) return EP_ERR_SCRATCH;
    if (dtype == EP_BF16) return dim == 64 ? launch<Bf16, 64>(P, st) : launch<Bf16, 128>(P, st);
    return dim == 64 ? launch<Fp16, 64>(P, st) : launch<Fp16, 128>(P, st);
}
