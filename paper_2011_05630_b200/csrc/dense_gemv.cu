// Forward products of a few tokens (at most 16): what bounds them is the weights' way from memory, and a tile of the larger
// kernels would be mostly empty rows behind a longer way (shared memory, tensor memory, an exchange).  Here the weights go from
// memory straight into the registers of warp-level matrix instructions (16 weight rows x 8 tokens x 16 of K; their rate is
// of no account at 16 bytes of weights a lane for two of them): the order of K within an instruction is free as long as both operands
// have the same, so that a lane's 8 consecutive values of a row are its share of two instructions, and nothing is rearranged.
//
// A CTA has a run of weight rows for itself, all CTAs one of the same length, two CTAs to an SM: every SM streams until the end.  Its
// eight warps share K in blocks of consecutive values and meet in shared memory, in the order of the warps.  Rows may start anywhere:
// off the 16-byte boundaries a lane takes the two aligned pieces that hold its values and shifts them together.
#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_mem.cuh"
#include "ptx.cuh"

namespace dlf {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

struct GemvParams {
    Mat x, w[2], o[3], res;
    const float* bias[2];
    long long N;
    int M, K, act, rows;   // rows: weight rows of a CTA
};

template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT: runs of 8 tokens.  ANY: rows start anywhere, or end inside 16 bytes.
template <typename T, int NT, bool GATED, bool ANY>
__global__ void __launch_bounds__(kThreads, 2) dense_gemv_kernel(const __grid_constant__ GemvParams p) {
    constexpr int NW = GATED ? 2 : 1;   // weight matrices
    constexpr int D = ANY ? (GATED || NT > 1 ? 2 : 3) : GATED ? (NT > 1 ? 3 : 4) : NT > 1 ? 5 : 6;   // steps of 32 of K that are on their way at a time
    __shared__ float part_s[2][kWarps][NW * 16][8 * NT + 2];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const long long first = static_cast<long long>(blockIdx.x) * p.rows, end = min(first + p.rows, p.N);
    // K goes round the warps in blocks of D steps (side by side: pieces of 64 bytes a row make the memory slower); the loads run a block ahead of the products, into the next 16 rows too
    const int blocks = ((p.K + 31) / 32 + kWarps * D - 1) / (kWarps * D);
    const unsigned short* x[NT];
#pragma unroll
    for (int j = 0; j < NT; j++) x[j] = static_cast<const unsigned short*>(p.x.p) + min(g + 8 * j, p.M - 1) * p.x.ld + t * 8;
    struct At {
        long long n0;
        const unsigned short* w[NW][2];
        bool live[2];
        int block;
    };
    auto rows_of = [&](At& a) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            a.live[h] = a.n0 + g + 8 * h < end;
#pragma unroll
            for (int q = 0; q < NW; q++) a.w[q][h] = static_cast<const unsigned short*>(p.w[q].p) + (a.live[h] ? a.n0 + g + 8 * h : first) * p.w[q].ld + t * 8;
        }
    };
    Eight<ANY, true> wv[D][NW][2];
    Eight<ANY, false> xv[D][NT];
    auto fetch = [&](const At& a, int d) {
        const int k = ((a.block * kWarps + warp) * D + d) * 32, n = p.K - k - t * 8;   // values that this lane's piece of the step has
#pragma unroll
        for (int q = 0; q < NW; q++)
#pragma unroll
            for (int h = 0; h < 2; h++) wv[d][q][h].fetch(a.w[q][h] + k, a.live[h] ? n : 0);
#pragma unroll
        for (int j = 0; j < NT; j++) xv[d][j].fetch(x[j] + k, g + 8 * j < p.M ? n : 0);
    };
    At ahead{first, {}, {}, 0};
    rows_of(ahead);
#pragma unroll
    for (int d = 0; d < D; d++) fetch(ahead, d);
    int buf = 0;
#pragma unroll 1
    for (long long n0 = first; n0 < end; n0 += 16, buf ^= 1) {
        float acc[NW][NT][4] = {};
#pragma unroll 1
        for (int block = 0; block < blocks; block++) {
            At now = ahead;
            if (++ahead.block == blocks) {
                ahead.block = 0;
                ahead.n0 += 16;
                rows_of(ahead);   // (past the last row: nothing is live)
            }
#pragma unroll
            for (int d = 0; d < D; d++) {
                uint4 c[NT];
                const int k = ((block * kWarps + warp) * D + d) * 32, n = p.K - k - t * 8;
#pragma unroll
                for (int j = 0; j < NT; j++) c[j] = xv[d][j].get(x[j] + k, g + 8 * j < p.M ? n : 0);
#pragma unroll
                for (int q = 0; q < NW; q++) {
                    const uint4 a = wv[d][q][0].get(now.w[q][0] + k, now.live[0] ? n : 0), b = wv[d][q][1].get(now.w[q][1] + k, now.live[1] ? n : 0);
#pragma unroll
                    for (int j = 0; j < NT; j++) {
                        mma16816<T>(acc[q][j], a.x, b.x, a.y, b.y, c[j].x, c[j].y);
                        mma16816<T>(acc[q][j], a.z, b.z, a.w, b.w, c[j].z, c[j].w);
                    }
                }
                fetch(ahead, d);
            }
        }
#pragma unroll
        for (int q = 0; q < NW; q++)
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    *reinterpret_cast<float2*>(&part_s[buf][warp][q * 16 + g + 8 * h][8 * j + 2 * t]) = make_float2(acc[q][j][2 * h], acc[q][j][2 * h + 1]);
        __syncthreads();   // (the other buffer is free again: who reads it has passed this)
        const int r = threadIdx.x & 15, m = threadIdx.x >> 4;   // a thread finishes one output
        const long long n = n0 + r;
        if (m < p.M && m < 8 * NT && n < end) {
            auto total = [&](int row) {
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < kWarps; i++) v += part_s[buf][i][row][m];
                return v;
            };
            auto put = [&](const Mat& o, float v) { static_cast<T*>(const_cast<void*>(o.p))[m * o.ld + n] = from_f32<T>(v); };
            float z = total(r);
            if (p.bias[0]) z += ld_map(p.bias[0] + n);
            if (GATED) {
                float u = total(GATED ? 16 + r : 0);
                if (p.bias[1]) u += ld_map(p.bias[1] + n);
                if (p.o[1].p) put(p.o[1], z);
                if (p.o[2].p) put(p.o[2], u);
                with_act(p.act, [&](auto act) { put(p.o[0], act_f<act.value>(z) * u); });
            } else {
                if (p.res.p) z += to_f32(ld_map(static_cast<const T*>(p.res.p) + m * p.res.ld + n));
                if (p.o[1].p) put(p.o[1], z);
                with_act(p.act, [&](auto act) { put(p.o[0], act_f<act.value>(z)); });
            }
        }
    }
}

typedef void (*GemvFn)(const GemvParams);
template <typename T, int NT>
GemvFn pick_gemv(bool gated, bool any) {
    if (gated) return any ? dense_gemv_kernel<T, NT, true, true> : dense_gemv_kernel<T, NT, true, false>;
    return any ? dense_gemv_kernel<T, NT, false, true> : dense_gemv_kernel<T, NT, false, false>;
}

}  // namespace

bool dense_gemv_takes(int64_t m) { return m <= 16; }

int launch_dense_gemv(const DenseGemm& g, cudaStream_t s) {
    int sms = 0;
    const int rc = query_sms(&sms);
    if (rc) return rc;
    GemvParams p{};
    p.x = g.a[0];
    for (int i = 0; i < 2; i++) { p.w[i] = g.b[i]; p.bias[i] = g.bias[i]; }
    for (int i = 0; i < 3; i++) p.o[i] = g.out[i];
    p.res = g.res;
    p.N = g.N; p.M = static_cast<int>(g.M); p.K = static_cast<int>(g.K); p.act = g.act;
    p.rows = static_cast<int>(std::max<int64_t>(8, (g.N + 2 * sms - 1) / (2 * sms)));
    const int grid = static_cast<int>((g.N + p.rows - 1) / p.rows);
    const bool bf = g.dtype == DLF_BF16, any = g.K % 8 != 0 || !dense_rows16(g.a[0]) || !dense_rows16(g.b[0]) || !dense_rows16(g.b[1]);
    const GemvFn fn = g.M > 8 ? (bf ? pick_gemv<__nv_bfloat16, 2>(g.gated, any) : pick_gemv<__half, 2>(g.gated, any))
                              : (bf ? pick_gemv<__nv_bfloat16, 1>(g.gated, any) : pick_gemv<__half, 1>(g.gated, any));
    const cudaError_t e = launch_kernel(fn, grid, kThreads, 0, s, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

}  // namespace dlf
