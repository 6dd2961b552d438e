// Pieces of 16 bytes of rows that start on 16-byte boundaries or anywhere.
#pragma once
#include <stdint.h>

#include "ptx.cuh"

namespace dlf {

// 16 bytes if `live`, else zeros: one predicated load, no branch.  Weights are read once: they do not push the tokens out of the
// first-level cache.
template <bool STREAM>
__device__ __forceinline__ uint4 ld16_if(const void* p, bool live) {
    uint4 v;
    if (STREAM)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                     "@q ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                     : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"(static_cast<int>(live)) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                     "@q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                     : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"(static_cast<int>(live)) : "memory");
    return v;
}

// 16 of the 32 bytes of two pieces, from byte s on (an even number below 16).
__device__ __forceinline__ uint4 shift16(const uint4& a, const uint4& b, uint32_t s) {
    uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, w[4];
#pragma unroll
    for (int i = 0; i < 6; i++) v[i] = s & 8 ? v[i + 2] : v[i];
#pragma unroll
    for (int i = 0; i < 5; i++) v[i] = s & 4 ? v[i + 1] : v[i];
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = s & 2 ? __funnelshift_r(v[i], v[i + 1], 16) : v[i];
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 8 consecutive values of a row from p on, n of which exist, zeros for the others: in one or two aligned pieces of 16 bytes (a piece that
// holds one of them lies in memory that exists).
__device__ __forceinline__ uint4 load8_any(const unsigned short* p, int n) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), s = at & 15;
    const uint4 a = ld16_if<true>(reinterpret_cast<const void*>(at - s), n > 0);
    const uint4 b = ld16_if<true>(reinterpret_cast<const void*>(at - s + 16), n > 0 && static_cast<int>(s) + 2 * min(n, 8) > 16);
    const uint4 q = shift16(a, b, static_cast<uint32_t>(s));
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = 2 * i + 1 < n ? w[i] : 2 * i < n ? w[i] & 0xffffu : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace dlf
