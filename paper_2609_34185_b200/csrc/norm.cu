// Norms before and after a block, fused with the block's gate and the residual, into a 16- or 32-bit type or an 8-bit container.
#include "op_rows.hpp"

using namespace ep;

namespace {

constexpr uint32_t kMaxColumns = 32768;

// ======================================================================================================================
//   b = norm(x) (o + p),   r = c h + g b,   z = norm(r) (o + w) + d,   norm(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps)
//
// A row stays in the registers of its warps from its first byte to its last: x and h are read once, r and z written once, whatever
// stands between.  Deviations from the mean are summed in a second walk through the registers, so that nothing cancels.
// Bound by memory for many rows, by the launch and two to five exchanges between warps for few.
// ======================================================================================================================
struct NormVector {
    const uint8_t *d;
    int64_t pitch;                // bytes between groups
    uint32_t rows;                // of a group
    int32_t dtype;
    uint32_t vec;
};
struct NormParams {
    const uint8_t *x, *h;
    uint8_t *r, *z, *s;
    int64_t ldx, ldh, ldr, ldz, lds;      // bytes; scales: elements
    NormVector w, d, g, p;
    float c, offset, eps, columns;
    uint32_t T, C;
    uint32_t warps, rows;         // warps of a row, rows of a CTA
    int32_t x_half, h_half, r_dtype, z_dtype, center;
    uint32_t x_vec, h_vec, r_vec, z_vec;
};

__device__ __forceinline__ void load_vector(const NormVector &V, uint32_t row, uint32_t c, uint32_t n, float (&v)[8]) {
    const uint8_t *at = V.d + int64_t(V.rows ? row / V.rows : 0) * V.pitch;
    if (V.dtype == EP_FP32) {
        Eight<32> e;
        load_eight<32, true>(at, c, n, V.vec, e);
        to_floats<32>(e, false, v);
    } else {
        Eight<16> e;
        load_eight<16, true>(at, c, n, V.vec, e);
        to_floats<16>(e, V.dtype == EP_FP16, v);
    }
}

// v becomes (v - mean) / sqrt(mean square of that + eps)
template <uint32_t N>
__device__ __forceinline__ void normed(const NormParams &P, RowGroup &group, const uint32_t (&n)[N], float (&v)[N][8]) {
    if (P.center) {
        float sum = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) sum += j < n[i] ? v[i][j] : 0.0f;
        const float mean = group.sum(sum) / P.columns;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[i][j] -= mean;
    }
    float squares = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) squares += j < n[i] ? v[i][j] * v[i][j] : 0.0f;
    const float f = 1.0f / sqrtf(group.sum(squares) / P.columns + P.eps);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) v[i][j] *= f;
}

template <uint32_t XBITS, uint32_t HBITS, uint32_t N, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS) norm_kernel(const __grid_constant__ NormParams P) {
    __shared__ uint32_t room[64];
    op_wait_for_stream();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, of = warp / P.warps;
    const uint32_t row = blockIdx.x * P.rows + of, l = (warp - of * P.warps) * 32u + lane;
    RowGroup group{room, P.warps, of * P.warps, 0};
    const bool there = row < P.T;
    Eight<XBITS> x[N];
    Eight<HBITS> h[N];
    uint32_t n[N];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t c = (i * P.warps * 32u + l) * 8u;
        n[i] = there ? inside(c, P.C) : 0u;
        load_eight<XBITS>(P.x + int64_t(row) * P.ldx, c, n[i], P.x_vec, x[i]);
        if (P.h) load_eight<HBITS>(P.h + int64_t(row) * P.ldh, c, n[i], P.h_vec, h[i]);
    }
    float v[N][8];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) to_floats<XBITS>(x[i], P.x_half, v[i]);
    if (P.p.d) {
        normed<N>(P, group, n, v);
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                float p[8];
                load_vector(P.p, row, (i * P.warps * 32u + l) * 8u, n[i], p);
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) v[i][j] *= P.offset + p[j];
            }
    }
    if (P.g.d)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            float g[8];
            load_vector(P.g, row, (i * P.warps * 32u + l) * 8u, n[i], g);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
    if (P.h)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            float old[8];
            to_floats<HBITS>(h[i], P.h_half, old);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[i][j] = fmaf(P.c, old[j], v[i][j]);
        }
    if (P.r)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) store_floats(P.r + int64_t(row) * P.ldr, (i * P.warps * 32u + l) * 8u, n[i], P.r_dtype, P.r_vec, v[i]);
    normed<N>(P, group, n, v);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t c = (i * P.warps * 32u + l) * 8u;
        if (P.w.d) {
            float w[8];
            load_vector(P.w, row, c, n[i], w);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[i][j] *= P.offset + w[j];
        }
        if (P.d.d) {
            float d[8];
            load_vector(P.d, row, c, n[i], d);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[i][j] += d[j];
        }
    }
    uint8_t *z = P.z + int64_t(row) * P.ldz;
    if (P.z_dtype == EP_INT8) {
        uint32_t top = 0;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) top = max(top, j < n[i] ? __float_as_uint(v[i][j]) & 0x7FFFFFFFu : 0u);
        const Int8Scale s = int8_scale(group.largest(top));
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            float q[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) q[j] = s.inverse == 0.0f ? 0.0f : __fmul_rn(v[i][j], s.inverse);
            store_bytes(z, (i * P.warps * 32u + l) * 8u, n[i], P.z_vec, int8x4(q[0], q[1], q[2], q[3]), int8x4(q[4], q[5], q[6], q[7]));
        }
        if (l == 0 && there) reinterpret_cast<float *>(P.s)[row] = s.s;
    } else if (P.z_dtype == EP_FP8_E4M3) {
        const float infinity = __uint_as_float(0x7F800000u);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {                               // a block of 128 values is sixteen lanes'
            const uint32_t c = (i * P.warps * 32u + l) * 8u;
            float top = 0.0f;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                const bool fine = fabsf(v[i][j]) < infinity;
                top = fmaxf(top, fine && j < n[i] ? fabsf(v[i][j]) : 0.0f);
                if (!fine) v[i][j] = __uint_as_float(0x7FFFFFFFu);
            }
#pragma unroll
            for (uint32_t m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
            const uint32_t e = scale_exponent(top, 127u);
            const float f = pow2_inverse(e);
            store_bytes(z, c, n[i], P.z_vec, e4m3x2(v[i][0] * f, v[i][1] * f) | e4m3x2(v[i][2] * f, v[i][3] * f) << 16,
                        e4m3x2(v[i][4] * f, v[i][5] * f) | e4m3x2(v[i][6] * f, v[i][7] * f) << 16);
            if ((lane & 15u) == 0 && n[i]) P.s[int64_t(row) * P.lds + c / 128u] = uint8_t(e);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) store_floats(z, (i * P.warps * 32u + l) * 8u, n[i], P.z_dtype, P.z_vec, v[i]);
    }
}

template <uint32_t XBITS, uint32_t HBITS>
int launch_norm(NormParams P, cudaStream_t st) {
    const uint32_t pieces = (P.C + 7u) / 8u;
    const uint32_t each = pieces <= 1024 ? 1u : pieces <= 2048 ? 4u : 8u;
    P.warps = (pieces + 32u * each - 1u) / (32u * each);
    P.rows = P.warps >= 4 ? 1u : 4u / P.warps;
    const uint32_t threads = P.warps * P.rows * 32u, grid = uint32_t((uint64_t(P.T) + P.rows - 1u) / P.rows);
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

int vector_of(const ep_vector &v, uint32_t T, uint32_t C, NormVector &out) {
    std::memset(&out, 0, sizeof(out));
    if (!v.d) return EP_OK;
    const uint32_t size = bytes_of(v.dtype);
    if (!size || v.groups == 0 || T % v.groups || !aligned(v.d, size) || (v.groups > 1 && !rows_fit(v.d, v.ld, C, size))) return EP_ERR_BAD_ARG;
    out.d = static_cast<const uint8_t *>(v.d);
    out.dtype = v.dtype;
    if (v.groups > 1) out.pitch = v.ld * size, out.rows = T / v.groups;
    out.vec = rows_begin_on(16, v.d, v.groups > 1 ? v.ld : 0, size);
    return EP_OK;
}

}  // namespace

extern "C" int ep_norm(const ep_norm_job *job, void *stream) {
    if (!job) return EP_ERR_BAD_ARG;
    const ep_norm_job &j = *job;
    if (j.T == 0) return EP_OK;
    const uint32_t xs = bytes_of(j.x_dtype), hs = bytes_of(j.residual_dtype), zs = j.z_dtype == EP_FP8_E4M3 || j.z_dtype == EP_INT8 ? 1u : bytes_of(j.z_dtype);
    const bool residual = j.d_residual || j.d_residual_out;
    if (!j.d_x || !j.d_z || j.C == 0 || j.T > 0x7FFFFF00u || !xs || !zs || (residual && !hs) || !rows_fit(j.d_x, j.ldx, j.C, xs) || !rows_fit(j.d_z, j.ldz, j.C, zs) ||
        (j.d_residual && !rows_fit(j.d_residual, j.ld_residual, j.C, hs)) || (j.d_residual_out && !rows_fit(j.d_residual_out, j.ld_residual_out, j.C, hs)) ||
        (j.d_residual && j.d_residual == j.d_residual_out && j.ld_residual != j.ld_residual_out))
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
    P.T = j.T;
    P.C = j.C;
    P.x_half = j.x_dtype == EP_FP16;
    P.h_half = j.residual_dtype == EP_FP16;
    P.r_dtype = j.residual_dtype;
    P.z_dtype = j.z_dtype;
    P.center = j.center != 0;
    P.x_vec = rows_begin_on(16, j.d_x, j.ldx, xs);
    P.h_vec = j.d_residual && rows_begin_on(16, j.d_residual, j.ld_residual, hs);
    P.r_vec = j.d_residual_out && rows_begin_on(16, j.d_residual_out, j.ld_residual_out, hs);
    P.z_vec = rows_begin_on(zs == 1 ? 8 : 16, j.d_z, j.ldz, zs);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (xs == 4) return j.d_residual && hs == 4 ? launch_norm<32, 32>(P, st) : launch_norm<32, 16>(P, st);
    return j.d_residual && hs == 4 ? launch_norm<16, 32>(P, st) : launch_norm<16, 16>(P, st);
}
