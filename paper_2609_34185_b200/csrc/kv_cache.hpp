// What the kernels of the paged cache share.
#pragma once
#include "op8.hpp"

namespace ep {

#ifdef __CUDACC__

// What both operators read: where the requests' tokens stand.  Request b has seq_lens[b] tokens in the cache, the last
// starts[b + 1] - starts[b] of which are its rows of the call; token j lies in page table[b][j / page], row j % page.
struct Requests {
    const int32_t *table, *seq_lens, *starts;
    int64_t ldt;
    uint32_t B, N, columns;       // requests; rows of the call; columns of the table
    uint32_t pages, page, shift;  // pages of the cache, tokens of a page = 1 << shift
    uint32_t H;                   // heads of the cache
};
// rows and tokens of request b; whatever the arrays hold, rows lie inside the call's and tokens inside the table
struct Extent { uint32_t row, rows, len; };
__host__ __device__ __forceinline__ int32_t entry_of(const int32_t *p) {
#ifdef __CUDA_ARCH__
    return __ldg(p);
#else
    return *p;
#endif
}
__host__ __device__ __forceinline__ Extent extent_of(const Requests &q, uint32_t b) {
    const uint32_t lo = uint32_t(min(max(entry_of(q.starts + b), 0), int32_t(q.N))), hi = uint32_t(min(max(entry_of(q.starts + b + 1), int32_t(lo)), int32_t(q.N)));
    const uint64_t room = uint64_t(q.columns) << q.shift;
    return {lo, hi - lo, uint32_t(min(uint64_t(uint32_t(max(entry_of(q.seq_lens + b), 0))), room))};
}

// The softmax's weights carry the pages' value scales, as ratios to one page's of the request: t = score + log2(ratio), and a row's sum
// takes them out again.  That page is the first one that is more than zeros (append leaves those with 2^-100, and a ratio to that would leave fp32's
// range).  What a weight would lose below fp32's range is lost to the sum, so ratios stop at 2^-60: the values of a page further below (zeros
// again) then count as up to 2^-51 of that page's largest, less than fp32 resolves, and weights keep 2^-30 of the largest for pages of
// up to 2^40 times that one's scale.
constexpr float kLeastRatio = 0x1p-60f;
// the value scale that ratios refer to: of the first page above 2^-100 (and below 2^120), else of the first page, else 1; by a whole warp
__device__ __forceinline__ float first_scale(const Requests &q, const float *vs, uint32_t b, uint32_t h, uint32_t len) {
    const int32_t *row = q.table + int64_t(b) * q.ldt;
    auto scale_at = [&](uint32_t j) {
        const int32_t id = __ldg(row + j);
        return uint32_t(id) < q.pages ? __ldg(vs + size_t(uint32_t(id)) * q.H + h) : 0.0f;
    };
    auto serves = [](float v, float least) { return v > least && v < 0x1p120f; };
    const float v = scale_at(0);
    if (serves(v, 0x1p-100f)) return v;
    const uint32_t lane = threadIdx.x & 31u, n = (len + q.page - 1u) >> q.shift;
#pragma unroll 1
    for (uint32_t j = 0; j < n; j += 32u) {
        const float other = j + lane < n ? scale_at(j + lane) : 0.0f;
        const uint32_t found = __ballot_sync(0xFFFFFFFFu, serves(other, 0x1p-100f));
        if (found) return __shfl_sync(0xFFFFFFFFu, other, __ffs(int(found)) - 1);
    }
    return serves(v, 0x1p-120f) ? v : 1.0f;
}

// ---- softmax in powers of two -------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// prefix[b] = the sum of units(b') over b' < b, prefix[B] = all; by a whole CTA of at most 32 warps.  Returns all, and 0 if that is
// more than `most`, which no call can come to whose requests' rows are its own: sums stop at 2^32 - 1 on the way.
__host__ __device__ __forceinline__ uint32_t add_capped(uint32_t a, uint32_t b) { return a + b < a ? 0xFFFFFFFFu : a + b; }
// A thread's requests b0 .. b1 - 1: the sum of their units, then, with what lies before them, their entries.
template <class F>
__host__ __device__ __forceinline__ uint32_t sum_units(uint32_t b0, uint32_t b1, F units) {
    uint32_t sum = 0;
    for (uint32_t b = b0; b < b1; ++b) sum = add_capped(sum, units(b));
    return sum;
}
template <class F>
__host__ __device__ __forceinline__ void lay_prefix(uint32_t b0, uint32_t b1, uint32_t at, F units, uint32_t *prefix) {
    for (uint32_t b = b0; b < b1; ++b) {
        const uint32_t n = units(b);                      // (the count may stand in prefix[b])
        prefix[b] = at;
        at += n;
    }
}
template <class F>
__device__ uint32_t prefix_sums(uint32_t B, F units, uint32_t most, uint32_t *prefix, uint32_t *part) {
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, per = (B + blockDim.x - 1u) / blockDim.x;
    const uint32_t b0 = min(tid * per, B), b1 = min(b0 + per, B);
    const uint32_t sum = sum_units(b0, b1, units);
    uint32_t inc = sum;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
        if (lane >= d) inc = add_capped(inc, o);
    }
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    uint32_t at = inc - sum, all = 0;
    for (uint32_t w = 0; w < (blockDim.x >> 5); ++w) {
        if (w < warp) at += part[w];
        all = add_capped(all, part[w]);
    }
    lay_prefix(b0, b1, at, units, prefix);
    if (tid == 0) prefix[B] = all;
    __syncthreads();
    return all <= most ? all : 0u;
}
// the last b in [lo, B) with prefix[b] <= u (prefix[lo] <= u < prefix[B]): its units hold u
__device__ __forceinline__ uint32_t request_of(const uint32_t *prefix, uint32_t lo, uint32_t B, uint32_t u) {
    uint32_t hi = B;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (prefix[mid] <= u) lo = mid; else hi = mid;
    }
    return lo;
}
constexpr uint32_t kMaxRequests = 4096;

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// two fp32 operations per instruction
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void pair_to(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

struct AttendParams {
    Requests q;
    const void *x;
    void *o;
    float *lse;                   // may be null
    const float *ks, *vs;
    const uint8_t *k, *v;
    int64_t ldq, ldqh, ldo, ldoh;
    uint32_t Hq, G;               // query heads; per head of the cache
    float scale_log2;             // scale * log2(e)
    uint32_t causal;
    float *workspace;             // null: no segment can cross a share
    uint32_t grid;
    uint32_t most;                // units (places) that a call of this size can come to
};

// many rows per request (attend_prompts.cu): whether a call's shape is for it; `cut`: segments may be cut (a workspace is there)
bool prompts_serve(uint32_t N, uint32_t B, uint32_t G);
size_t prompts_workspace_bytes(uint32_t grid, uint32_t dim);
int launch_prompts(AttendParams P, size_t workspace_bytes, bool cut, uint32_t dim, int32_t dtype, cudaStream_t st);

#endif  // __CUDACC__

}  // namespace ep
