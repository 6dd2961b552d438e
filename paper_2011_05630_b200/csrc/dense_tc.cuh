// What the tensor-core kernels of the dense operators share: tensor maps over row-major 16-bit matrices, products of a 64-value chunk
// of K with operands along or across K, rows of 64 values between registers and memory, and the word that a wait which gave up
// leaves its code in.
#pragma once
#include <cuda.h>

#include <atomic>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_mem.cuh"
#include "ptx.cuh"

namespace dlf {

// One for each source file that includes this (see dense_status_of).
static __device__ int g_dense_status;

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

// Waits for the stream and reads the status word; a code in it is reported once.
inline int dense_status_of(cudaStream_t s, int* code) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(code, g_dense_status, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return cuda_fail(e);
    if (*code) {
        const int zero = 0;
        e = cudaMemcpyToSymbolAsync(g_dense_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    return DLF_OK;
}

// ---- device ----------------------------------------------------------------------------------------------------------------
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

// A warp's 32 rows of 64 values from column col0 on, as they lie in memory, a lane its row: the first `cols` of them and, behind
// those and the matrix's last row, zeros.  Rows that start off the 16-byte boundaries, or end between two, come through `stg`
// (4096 bytes of the warp's own), whole runs of columns at a time.
template <typename T>
__device__ __forceinline__ void load_rows64(const Mat& m, bool vec, uint8_t* stg, int lane, int64_t row0, int64_t col0, int64_t rows_end, int cols, uint4 (&q)[8]) {
    const unsigned short* p = static_cast<const unsigned short*>(m.p) + row0 * m.ld + col0;
    const int rows = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(32), rows_end - row0)));
    if (vec && (cols & 7) == 0) {
        p += lane * m.ld;
#pragma unroll
        for (int j = 0; j < 8; j++) q[j] = lane < rows && j * 8 < cols ? ld_map(reinterpret_cast<const uint4*>(p + j * 8)) : make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    if (lane == 0) tma_store_wait_read();   // what lay here before has left
    __syncwarp();
#pragma unroll 8
    for (int r = 0; r < 32; r++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int c = lane + h * 32;
            const unsigned short v = r < rows && c < cols ? ld_map(p + r * m.ld + c) : static_cast<unsigned short>(0);
            *reinterpret_cast<unsigned short*>(stg + r * 128 + (((c >> 3) ^ (r & 7)) << 4) + (c & 7) * 2) = v;
        }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; j++) q[j] = *reinterpret_cast<const uint4*>(stg + lane * 128 + ((j ^ (lane & 7)) << 4));
    __syncwarp();
}
template <typename T>
__device__ __forceinline__ void add_row64(const uint4 (&q)[8], float* v) {
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const T* e = reinterpret_cast<const T*>(&q[j]);
#pragma unroll
        for (int i = 0; i < 8; i++) v[j * 8 + i] += to_f32(e[i]);
    }
}
__device__ __forceinline__ void add_bias64(const float* bias, int64_t col0, int cols, float* v) {
    const float* b = bias + col0;
    if (cols == 64 && (reinterpret_cast<uintptr_t>(b) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const float4 f = ld_map(reinterpret_cast<const float4*>(b) + i);
            v[4 * i] += f.x; v[4 * i + 1] += f.y; v[4 * i + 2] += f.z; v[4 * i + 3] += f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 64; i++)
            if (i < cols) v[i] += ld_map(b + i);
    }
}

// A warp's 32 rows of 64 values (a lane holds a row): rounded, through `stg` (4096 bytes of the warp's own) and out, by a TMA store
// where the output has a map, else row by row.  Rows and columns beyond the matrix are not written.  (A TMA store clips at the map's
// edge in pieces of 16 bytes: with a last piece that is not whole it writes zeros behind the row's end.)
template <typename T>
__device__ __forceinline__ void store_rows64(const Mat& o, const CUtensorMap* map, bool tma, uint8_t* stg, int lane, int64_t row0, int64_t col0,
                                             int64_t rows_end, int cols, const float* v) {
    if (lane == 0) tma_store_wait_read();   // what lay here before has left
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const uint4 q = make_uint4(pack2<T>(v[8 * j], v[8 * j + 1]), pack2<T>(v[8 * j + 2], v[8 * j + 3]), pack2<T>(v[8 * j + 4], v[8 * j + 5]),
                                   pack2<T>(v[8 * j + 6], v[8 * j + 7]));
        *reinterpret_cast<uint4*>(stg + lane * 128 + ((j ^ (lane & 7)) << 4)) = q;
    }
    if (tma && (cols & 7) == 0) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map, stg, static_cast<int>(col0), static_cast<int>(row0));
            tma_store_commit();
        }
    } else {
        __syncwarp();
        // a row's runs of 8 values begin where memory's pieces of 16 bytes do: nine runs a row, the first and the last not whole
        const int rows = static_cast<int>(min(static_cast<int64_t>(32), rows_end - row0));
        unsigned short* const p0 = static_cast<unsigned short*>(const_cast<void*>(o.p)) + row0 * o.ld + col0;
#pragma unroll 3
        for (int it = 0; it < 9; it++) {
            const int i = it * 32 + lane, r = i / 9;
            unsigned short* const p = p0 + r * o.ld;
            const int c = (i - r * 9) * 8 - static_cast<int>((reinterpret_cast<uintptr_t>(p) >> 1) & 7);   // its first column
            if (r >= rows || c >= cols || c + 8 <= 0) continue;
            const uint8_t* const row = stg + r * 128;
            if (c >= 0 && c + 8 <= cols) {
                const int k = c >> 3;
                const uint4 a = *reinterpret_cast<const uint4*>(row + ((k ^ (r & 7)) << 4)), b = *reinterpret_cast<const uint4*>(row + (((k + 1) & 7) ^ (r & 7)) * 16);
                *reinterpret_cast<uint4*>(p + c) = shift16(a, b, static_cast<uint32_t>(c & 7) * 2);
            } else {
                for (int e = max(0, -c); e < 8 && c + e < cols; e++)
                    p[c + e] = *reinterpret_cast<const unsigned short*>(row + ((((c + e) >> 3) ^ (r & 7)) << 4) + ((c + e) & 7) * 2);
            }
        }
        __syncwarp();
    }
}

}  // namespace dlf
