// Dense products on the CUDA cores: 64 x 64 tiles of the result, 16 of K at a time in shared memory, 4 x 4 sums in fp32 per thread.
// Any strides and sizes.
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "ptx.cuh"

namespace dlf {

namespace {

constexpr int kTile = 64, kStep = 16;

template <typename T>
__device__ __forceinline__ float elem(const Mat& m, bool mn, int64_t i, int64_t k) {
    return to_f32(ld_map(static_cast<const T*>(m.p) + (mn ? k * m.ld + i : i * m.ld + k)));
}

template <typename T>
__global__ void __launch_bounds__(256) dense_simt_kernel(const __grid_constant__ DenseGemm g, int tiles_n, int64_t tiles) {
    __shared__ float as[kStep][kTile + 4], bs[2][kStep][kTile + 4];
    pdl_wait();
    pdl_launch_dependents();
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int n_b = g.gated ? 2 : 1;
    for (int64_t work = blockIdx.x; work < tiles * g.groups; work += gridDim.x) {
        const int group = work >= tiles ? 1 : 0;
        const int64_t t = work - group * tiles, m0 = t / tiles_n * kTile, n0 = t % tiles_n * kTile;
        float acc[2][4][4] = {};
        for (int src = 0; src < g.sources; src++) {
            const Mat& a = g.a[g.groups > 1 ? group : src];
            for (int64_t k0 = 0; k0 < g.K; k0 += kStep) {
                for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
                    const int ka = g.a_mn ? i / kTile : i % kStep, ma = g.a_mn ? i % kTile : i / kStep;
                    as[ka][ma] = m0 + ma < g.M && k0 + ka < g.K ? elem<T>(a, g.a_mn, m0 + ma, k0 + ka) : 0.0f;
                    const int kb = g.b_mn ? i / kTile : i % kStep, nb = g.b_mn ? i % kTile : i / kStep;
                    const bool in = n0 + nb < g.N && k0 + kb < g.K;
                    for (int j = 0; j < n_b; j++) bs[j][kb][nb] = in ? elem<T>(g.b[g.gated ? j : src], g.b_mn, n0 + nb, k0 + kb) : 0.0f;
                }
                __syncthreads();
                for (int k = 0; k < kStep; k++) {
                    float av[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) av[i] = as[k][ty * 4 + i];
                    for (int j = 0; j < n_b; j++)
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const float bv = bs[j][k][tx * 4 + c];
#pragma unroll
                            for (int i = 0; i < 4; i++) acc[j][i][c] += av[i] * bv;
                        }
                }
                __syncthreads();
            }
        }
        with_act(g.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + c;
                    if (m >= g.M || n >= g.N) continue;
                    auto put = [&](const Mat& o, float v) {
                        if (o.p) static_cast<T*>(const_cast<void*>(o.p))[m * o.ld + n] = from_f32<T>(v);
                    };
                    float z = acc[0][i][c];
                    if (g.bias[0]) z += g.bias[0][n];
                    if (g.gated) {
                        float u = acc[1][i][c];
                        if (g.bias[1]) u += g.bias[1][n];
                        put(g.out[0], act_f<act.value>(z) * u);
                        put(g.out[1], z);
                        put(g.out[2], u);
                    } else if (g.groups > 1) {
                        put(g.out[group], z);
                    } else {
                        if (g.res.p) z += to_f32(ld_map(static_cast<const T*>(g.res.p) + m * g.res.ld + n));
                        put(g.out[0], act_f<act.value>(z));
                        put(g.out[1], z);
                    }
                }
            }
        });
    }
}

}  // namespace

int launch_dense_simt(const DenseGemm& g, cudaStream_t s) {
    int sms = 0;
    const int rc = query_sms(&sms);
    if (rc) return rc;
    const int64_t tiles_n = (g.N + kTile - 1) / kTile, tiles = tiles_n * ((g.M + kTile - 1) / kTile);
    const int grid = static_cast<int>(std::min<int64_t>(tiles * g.groups, 4ll * sms));
    const cudaError_t e = g.dtype == DLF_BF16 ? launch_kernel(dense_simt_kernel<__nv_bfloat16>, grid, 256, 0, s, g, static_cast<int>(tiles_n), tiles)
                                              : launch_kernel(dense_simt_kernel<__half>, grid, 256, 0, s, g, static_cast<int>(tiles_n), tiles);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

}  // namespace dlf
