// What the tensor-core kernels of the dense operators share: tensor maps over row-major 16-bit matrices, products of a 64-value chunk
// of K with operands along or across K, and the word that a wait which gave up leaves its code in.
#pragma once
#include <cuda.h>

#include <atomic>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_mem.cuh"
#include "ptx.cuh"

namespace dlf {

// Where a bounded wait first gave up, and the number of CTAs in which one has so far: never cleared, so that no report can take another's.  One for
// each source file that includes this: what names it is static.
static __device__ int g_dense_status[2];

// ---- host ------------------------------------------------------------------------------------------------------------------
// A map over a matrix of `rows` rows of `cols` values (any 16-bit type: the copies move bits), boxes of box_rows x box_cols.
inline int dense_map(CUtensorMap* m, const Mat& a, int64_t rows, int64_t cols, int box_rows, int box_cols) {
    const uint64_t dims[2] = {static_cast<uint64_t>(cols), static_cast<uint64_t>(rows)};
    const uint64_t strides[1] = {static_cast<uint64_t>(a.ld) * 2};
    const uint32_t box[2] = {static_cast<uint32_t>(box_cols), static_cast<uint32_t>(box_rows)}, es[2] = {1, 1};
    return encode_tmap(m, a.p, 2, dims, strides, box, es);
}

// Raises a kernel's limit of dynamic shared memory once per device.
inline int dense_smem_attr(const void* fn, int bytes) {
    constexpr int kMax = 64;
    static std::atomic<const void*> seen[kMaxDevices][kMax];
    const int dev = current_device_slot();
    if (dev < 0) return DLF_E_UNSUPPORTED;
    int i = 0;
    for (; i < kMax; i++) {
        const void* f = seen[dev][i].load(std::memory_order_acquire);
        if (f == fn) return DLF_OK;
        if (!f) break;
    }
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return cuda_fail(e);
    const void* none = nullptr;
    if (i < kMax) seen[dev][i].compare_exchange_strong(none, fn, std::memory_order_release);   // (lost to another thread: set again next time)
    return DLF_OK;
}

// Waits for the stream and reads the number of CTAs in which a wait has given up.
static int dense_gave_up(cudaStream_t s, int* count) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_dense_status, sizeof(int), sizeof(int), cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

// ---- device ----------------------------------------------------------------------------------------------------------------
// At a CTA's end, by one thread.
static __device__ __forceinline__ void dense_count_abort() { atomicAdd(&g_dense_status[1], 1); }

// A wait at a barrier that nothing arrives at, as the kernels wait (see dlf_dense_debug_stall).
static __global__ void dense_stall_kernel(unsigned long long limit_ns) {
    __shared__ uint64_t bar;
    __shared__ int abort_s;
    if (threadIdx.x == 0) {
        abort_s = 0;
        mbar_init(&bar, 1);
        fence_barrier_init();
    }
    __syncthreads();
    mbar_wait(&bar, 0u, &abort_s, g_dense_status, 0xf00, limit_ns);
    __syncthreads();
    if (abort_s && threadIdx.x == 0) dense_count_abort();
}
static int dense_stall(unsigned long long limit_ns, cudaStream_t s) {
    dense_stall_kernel<<<1, 64, 0, s>>>(limit_ns);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

// Instruction descriptor: fp16 or bf16 operands (bits 7 and 10), fp32 sums; bits 15 and 16: operand A, B across K.
template <typename T>
__host__ __device__ constexpr uint32_t dense_idesc(int m, int n, bool amn, bool bmn) {
    return (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | (amn ? 1u << 15 : 0u) | (bmn ? 1u << 16 : 0u) |
           (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

// The four K = 16 steps of a 64-value chunk in one statement.  Along K a step is 32 bytes further (2 units), across K two
// 1024-byte atoms (128 units).
#define DLF_DENSE_STEP(CG, S)                                                                                                  \
    "mad.lo.u32 ta, %6, " #S ", %1;\n\tmad.lo.u32 tb, %7, " #S ", %2;\n\tmov.b64 da, {ta, %5};\n\tmov.b64 db, {tb, %5};\n\t"     \
    "tcgen05.mma.cta_group::" #CG ".kind::f16 [%0], da, db, %3, p;\n\t"
#define DLF_DENSE_CHUNK(CG)                                                                                                    \
    "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t.reg .b32 ta, tb;\n\tsetp.ne.b32 p, %4, 0;\n\t" DLF_DENSE_STEP(CG, 0)             \
    "setp.eq.b32 p, %3, %3;\n\t" DLF_DENSE_STEP(CG, 1) DLF_DENSE_STEP(CG, 2) DLF_DENSE_STEP(CG, 3) "}"
template <int CG, bool AMN, bool BMN>
__device__ __forceinline__ void umma_chunk(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    if (CG == 2)
        asm volatile(DLF_DENSE_CHUNK(2)::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHiSw128), "n"(AMN ? 128 : 2), "n"(BMN ? 128 : 2) : "memory");
    else
        asm volatile(DLF_DENSE_CHUNK(1)::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHiSw128), "n"(AMN ? 128 : 2), "n"(BMN ? 128 : 2) : "memory");
}
#undef DLF_DENSE_STEP
#undef DLF_DENSE_CHUNK

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, const void* src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(src)), "r"(c0), "r"(c1) : "memory");
}

}  // namespace dlf
