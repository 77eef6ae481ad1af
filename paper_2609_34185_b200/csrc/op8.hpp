// What the kernels around the 8-bit containers share: E4M3 and power-of-two scales, 16-bit element types, mbarriers with
// bounded waits, and the launch that may overlap the kernel before it.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>
#include <type_traits>

#include "entropack.h"
#include "stream.hpp"

namespace ep {

#ifdef __CUDACC__

constexpr uint32_t kOpSpinLimit = 1u << 18;      // attempts of about a microsecond each before a wait gives up

// ---- numbers ---------------------------------------------------------------------------------------------------------
// The smallest power of two s with amax <= 448 s, as a biased exponent, at least 1 (2^-126): amax = m 2^e with 1 <= m < 2
// and 448 = 1.75 * 2^8, so s = 2^(e - 8) if m <= 1.75, else 2^(e - 7).  `zero` for an amax of 0.
__device__ __forceinline__ uint32_t scale_exponent(float amax, uint32_t zero) {
    const uint32_t u = __float_as_uint(amax);
    const int32_t e = int32_t(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return u == 0 ? zero : uint32_t(max(e, 1));
}
__device__ __forceinline__ float pow2_biased(uint32_t e) { return __uint_as_float(e << 23); }            // 2^(e - 127), 1 <= e <= 254
__device__ __forceinline__ float pow2_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }  // its reciprocal, 1 <= e <= 253

// two values to E4M3, the nearer, ties to even; beyond +-448 stays +-448, NaN becomes 0x7F
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// four E4M3 values as binary16, exactly (0x7F and 0xFF become NaN)
__device__ __forceinline__ void f16x4_of_e4m3x4(uint32_t four, uint32_t &lo, uint32_t &hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(four));
}

struct Bf16 {
    using T = __nv_bfloat16;
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
    static __device__ __forceinline__ T of(float f) { return __float2bfloat16_rn(f); }
    static __device__ __forceinline__ float to(T v) { return __bfloat162float(v); }
    static __device__ __forceinline__ uint32_t bits(T v) { return __bfloat16_as_ushort(v); }
    static __device__ __forceinline__ float of_bits(uint32_t b) { return __uint_as_float(b << 16); }
    static __device__ __forceinline__ uint32_t two(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
struct Fp16 {
    using T = __half;
    static __device__ __forceinline__ float lo(uint32_t w) { return __half2float(__ushort_as_half(uint16_t(w))); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __half2float(__ushort_as_half(uint16_t(w >> 16))); }
    static __device__ __forceinline__ T of(float f) { return __float2half_rn(f); }
    static __device__ __forceinline__ float to(T v) { return __half2float(v); }
    static __device__ __forceinline__ uint32_t bits(T v) { return __half_as_ushort(v); }
    static __device__ __forceinline__ float of_bits(uint32_t b) { return __half2float(__ushort_as_half(uint16_t(b))); }
    static __device__ __forceinline__ uint32_t two(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
struct Fp32 {
    using T = float;
    static __device__ __forceinline__ T of(float f) { return f; }
    static __device__ __forceinline__ float to(T v) { return v; }
    static __device__ __forceinline__ uint32_t bits(T v) { return __float_as_uint(v); }
    static __device__ __forceinline__ float of_bits(uint32_t b) { return __uint_as_float(b); }
};

// ---- shared memory, barriers -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t ld_smem(uint32_t a) {
    uint32_t v;
    asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void st_smem(uint32_t a, uint32_t v) { asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ uint4 ld_smem16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// one attempt; the hardware may hold the thread for up to about a microsecond
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
    return ok != 0;
}
// waits for the phase of this parity to end; false, and the CTA's abort word set, if it does not within the limit
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t abort_word) {
#pragma unroll 1
    for (uint32_t i = 0; i < kOpSpinLimit; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63u) == 63u && ld_smem(abort_word)) return false;
    }
    st_smem(abort_word, 1u);
    return false;
}
// the same for the end of a kernel whose abort word may be set already: what is in flight gets its time to land
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < kOpSpinLimit; ++i)
        if (bar_try(bar, parity)) return;
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}


// ---- tensor cores ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The warp that issues matrix instructions runs as a whole and one elected lane of it issues: its addresses then stay in uniform
// registers (issued from a branch of one lane, each instruction took some 150 cycles to be put together).
__device__ __forceinline__ uint32_t elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t lead) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(lead) : "memory");
}
// bar_wait by a whole warp, the same answer for all of it
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, uint32_t abort_word) { return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity, abort_word)); }
// Operands of rows of 128 bytes with 128-byte swizzle, groups of eight rows 1024 bytes apart.  K-major: a row is a row of the
// operand.  MN-major: a row is one k, its 128 bytes 64 16-bit values along M or N; `lead` bytes to the next 64 of those.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lead = 16) {
    return uint64_t((addr >> 4) & 0x3FFFu) | (uint64_t(lead >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
#define EP_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define EP_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// a warp's quarter of tensor memory: lane = row, registers = columns.  Loads are complete after tc_loaded, stores after tc_stored
__device__ __forceinline__ void tc_load16(uint32_t tmem, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : EP_R8(v, 0), EP_R8(v, 8) : "r"(tmem));
}
__device__ __forceinline__ void tc_load32(uint32_t tmem, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
                 "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : EP_R8(v, 0), EP_R8(v, 8), EP_R8(v, 16), EP_R8(v, 24) : "r"(tmem));
}
// the same, and what uses v comes after it
#define EP_U8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
__device__ __forceinline__ void tc_loaded32(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : EP_U8(v, 0), EP_U8(v, 8), EP_U8(v, 16), EP_U8(v, 24)::"memory");
}
__device__ __forceinline__ void tc_loaded16(uint32_t (&v)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : EP_U8(v, 0), EP_U8(v, 8)::"memory"); }
__device__ __forceinline__ void tc_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_store16(uint32_t tmem, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::EP_I8(v, 0), EP_I8(v, 8), "r"(tmem) : "memory");
}
__device__ __forceinline__ void tc_store32(uint32_t tmem, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::EP_I8(v, 0), EP_I8(v, 8), EP_I8(v, 16), EP_I8(v, 24), "r"(tmem) : "memory");
}
__device__ __forceinline__ void tc_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ends when everything earlier in the stream has; before it nothing is read or written
__device__ __forceinline__ void op_wait_for_stream() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ---- host ------------------------------------------------------------------------------------------------------------
// A launch that may come up while the kernel before it still runs (`kernel` begins with op_wait_for_stream), in clusters of
// `cluster` CTAs.
template <class... A>
inline cudaError_t op_launch(void (*kernel)(A...), dim3 grid, uint32_t threads, uint32_t smem, uint32_t cluster, cudaStream_t st, const A &...args) {
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// the shared-memory attribute of a kernel, set once per device
template <class K>
inline int op_configure(K kernel, uint32_t smem, bool (&done)[64]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return EP_ERR_CUDA;
    if (dev >= 0 && dev < 64 && done[dev]) return EP_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return EP_ERR_CUDA;
    if (dev >= 0 && dev < 64) done[dev] = true;
    return EP_OK;
}

// the value of a translation unit's integrity word, cleared if it is set; negative on a CUDA error
template <class W>
inline int op_status(W &word) {
    unsigned int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, word, sizeof(v)) != cudaSuccess) return -1;
    if (v && cudaMemcpyToSymbol(word, &zero, sizeof(zero)) != cudaSuccess) return -1;
    return int(v);
}

inline int op_sms() {
    static int sms[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64 && sms[dev]) return sms[dev];
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) sms[dev] = n;
    return n;
}

using TensorMapFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline TensorMapFn tensor_map_fn() {
    static TensorMapFn fn = nullptr;
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &res) != cudaSuccess || !p ||
            res != cudaDriverEntryPointSuccess)
            return nullptr;
        fn = reinterpret_cast<TensorMapFn>(p);
    }
    return fn;
}
// bytes [rows][cols], rows `pitch` bytes apart, as boxes of box_cols x box_rows; what lies outside arrives as zeros
inline int byte_map(CUtensorMap *map, const void *base, uint64_t cols, uint64_t rows, uint64_t pitch, uint32_t box_cols, uint32_t box_rows,
                    CUtensorMapSwizzle swizzle) {
    const TensorMapFn fn = tensor_map_fn();
    if (!fn) return EP_ERR_CUDA;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_cols, box_rows}, estr[2] = {1u, 1u};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? EP_OK : EP_ERR_CUDA;
}

#endif  // __CUDACC__

}  // namespace ep
