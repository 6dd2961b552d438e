// Dense products for results that do not fill the chip with the pairs' 256 x 256 tiles (dense_tc.cu): few tokens, where the
// weights have to be streamed through as many SMs as there are, narrow layers, short batches.  One tile of at most 128 x BN of the
// result per CTA, nothing persistent, and K shared out over a cluster of SPLIT CTAs that work on the same tile.
//
// The partial sums of a cluster meet in distributed shared memory: CTA d finishes every SPLIT-th run of the tile's rows; each warp
// sends the rows that it drained straight to the CTA that they belong to, a barrier there counts the bytes (st.async), and the
// ranks are added up in their order: no scratch in global memory, no atomics, the same bits every time.
//
// What the tile does not have costs nothing: a token tile of r rows loads r rows (the tensor core multiplies what lies behind them
// in shared memory too; those rows of the accumulator are not read).
//
// A cluster's CTAs wait for one another while they hold tensor memory, so one that shares an SM with another kernel's
// that waits for tensor memory in the same way could wait for ever: a cluster kernel takes enough shared memory to have its SM for itself.
#include <cuda.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_tc.cuh"

namespace dlf {

namespace {

constexpr int kEpiWarps = 8;                 // warps 0..7: warp & 3 = TMEM lane quarter, warp >> 2 = every other run of columns
constexpr int kProdWarp0 = kEpiWarps, kProdWarps = 3;   // warp w loads ring stages w, w + 3, ...
constexpr int kMmaWarp = kProdWarp0 + kProdWarps;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kMaxBN = 128, kMaxStages = 12;
constexpr int kMaxDynSmem = 225 * 1024;
constexpr int kAloneSmem = 200 * 1024;       // more than this leaves no room for another tensor-core kernel's CTA on the SM
enum { EPI_PLAIN = 0, EPI_LINEAR = 1, EPI_GATED = 2 };

struct LatParams {
    CUtensorMap a[2], b[2];
    Mat o[3], res;
    const float* bias[2];
    long long M, N;
    int tiles_n, BN, rows;             // rows: of A in a tile
    long long group_tiles;
    int chunks1, total, share;         // 64-value chunks of K: of the first source, of both, of a CTA
    int stages, a_bytes, stage_bytes, red_off, rows_per;
    int act, groups;
    bool vec[3], res_vec;              // rows on 16-byte boundaries
};

// The finished sums of 8 outputs of a row to memory.
template <typename T>
__device__ __forceinline__ void put8(const Mat& o, bool vec, long long row, long long col, int n, const float (&v)[8]) {
    T* p = static_cast<T*>(const_cast<void*>(o.p)) + row * o.ld + col;
    if (vec && n == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}
template <int EPI, typename T>
__device__ __forceinline__ void finish8(const LatParams& p, int group, long long row, long long col, float (&v)[8], float (&u)[8]) {
    const int n = static_cast<int>(min(8ll, p.N - col));
    if (EPI == EPI_PLAIN) {
        put8<T>(p.o[group], p.vec[group], row, col, n, v);
        return;
    }
    if (p.bias[0]) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += i < n ? ld_map(p.bias[0] + col + i) : 0.0f;
    }
    if (EPI == EPI_LINEAR) {
        if (p.res.p) {
            const T* r = static_cast<const T*>(p.res.p) + row * p.res.ld + col;
            if (p.res_vec && n == 8) {
                const uint4 q = ld_map(reinterpret_cast<const uint4*>(r));
                const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] += to_f32(e[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] += i < n ? to_f32(ld_map(r + i)) : 0.0f;
            }
        }
        if (p.o[1].p) put8<T>(p.o[1], p.vec[1], row, col, n, v);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act_f<act.value>(v[i]);
        });
    } else {
        if (p.bias[1]) {
#pragma unroll
            for (int i = 0; i < 8; i++) u[i] += i < n ? ld_map(p.bias[1] + col + i) : 0.0f;
        }
        if (p.o[1].p) put8<T>(p.o[1], p.vec[1], row, col, n, v);
        if (p.o[2].p) put8<T>(p.o[2], p.vec[2], row, col, n, u);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act_f<act.value>(v[i]) * u[i];
        });
    }
    put8<T>(p.o[0], p.vec[0], row, col, n, v);
}

template <typename T, bool AMN, bool BMN, int EPI, int SPLIT>
__global__ void __cluster_dims__(SPLIT, 1, 1) __launch_bounds__(kThreads, 1) dense_lat_kernel(const __grid_constant__ LatParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar, red_bar;
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s, red_abort_s;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sbase = smem_raw + (base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &abort_s;
    int* status = &g_dense_status;
    const int rank = SPLIT > 1 ? static_cast<int>(cluster_rank()) : 0;
    long long tile = static_cast<long long>(blockIdx.x) / SPLIT;
    const int group = p.groups > 1 && tile >= p.group_tiles ? 1 : 0;
    tile -= group ? p.group_tiles : 0;
    const long long tm = tile / p.tiles_n;
    const long long n0 = (tile - tm * p.tiles_n) * (EPI == EPI_GATED ? p.BN / 2 : p.BN), m0 = tm * p.rows;
    const int k_first = rank * p.share, k_count = min(p.share, p.total - k_first);
    const int live = static_cast<int>(min(static_cast<long long>(p.rows), p.M - m0));   // rows of the tile that exist

    if (warp == kProdWarp0) {
        if (lane < kMaxStages) {
            mbar_init(&full_bar[lane], 1);
            mbar_init(&empty_bar[lane], 1);
        }
        if (lane == 0) {
            abort_s = 0;
            red_abort_s = 0;
            mbar_init(&tfull_bar, 1);
            mbar_init(&red_bar, 1);
        }
        fence_barrier_init();
        // the bytes that the cluster's CTAs will send here (before the cluster's barrier, which every sender waits for)
        if (SPLIT > 1 && lane == 0) mbar_expect_tx(&red_bar, static_cast<uint32_t>(SPLIT * max(0, min(p.rows_per, live - rank * p.rows_per)) * p.BN) * 4u);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&tmem_base_s, kMaxBN);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (SPLIT > 1) cluster_arrive();   // all CTAs of the cluster run (waited for before rows go to the others)
    tc_fence_after_sync();
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t tmem_base = tmem_base_s;

    if (warp >= kProdWarp0 && warp < kMmaWarp) {
        // ---- producers: lane i issues a stage's i-th box, those of A first ----
        const int w = warp - kProdWarp0;
        const int boxes_a = AMN ? 2 : 1, boxes = boxes_a + (EPI == EPI_GATED ? 2 : BMN ? p.BN / 64 : 1);
        const uint32_t stage_tx = static_cast<uint32_t>(p.a_bytes + p.BN * 128);
        int turn = 0, st = 0;
        uint32_t ph = 1;
#pragma unroll 1
        for (int i = 0; i < k_count; i++) {
            if (turn == w) {
                if (i >= p.stages && !mbar_wait_warp<true>(&empty_bar[st], ph, abort_flag, status, 0xA00 | (blockIdx.x << 12))) break;
                if (lane == 0) mbar_expect_tx(&full_bar[st], stage_tx);
                __syncwarp();
                if (lane < boxes) {
                    const int c = k_first + i;
                    const bool second = c >= p.chunks1;
                    const int k0 = (second ? c - p.chunks1 : c) * 64, j = lane - boxes_a;
                    uint8_t* dst = sbase + st * p.stage_bytes;
                    if (j < 0) {
                        const CUtensorMap* map = &p.a[second || group ? 1 : 0];
                        if (AMN) tma_load_2d(dst + lane * 8192, map, &full_bar[st], static_cast<int>(m0) + lane * 64, k0);
                        else tma_load_2d(dst, map, &full_bar[st], k0, static_cast<int>(m0));
                    } else {
                        dst += p.a_bytes;
                        if (EPI == EPI_GATED) tma_load_2d(dst + j * p.BN * 64, &p.b[j], &full_bar[st], k0, static_cast<int>(n0));
                        else if (BMN) tma_load_2d(dst + j * 8192, &p.b[second ? 1 : 0], &full_bar[st], static_cast<int>(n0) + j * 64, k0);
                        else tma_load_2d(dst, &p.b[second ? 1 : 0], &full_bar[st], k0, static_cast<int>(n0));
                    }
                }
                __syncwarp();
            }
            if (++turn == kProdWarps) turn = 0;
            if (++st == p.stages) { st = 0; turn = 0; ph ^= 1u; }
        }
    } else if (warp == kMmaWarp) {
        const uint32_t idesc = dense_idesc<T>(128, 0, AMN, BMN) | (static_cast<uint32_t>(p.BN >> 3) << 17);
        const uint32_t a0 = AMN ? umma_desc_mn_lo(base, 8192) : umma_desc_lo(base);
        const uint32_t b0 = BMN ? umma_desc_mn_lo(base + p.a_bytes, 8192) : umma_desc_lo(base + p.a_bytes);
        const uint32_t stage16 = static_cast<uint32_t>(p.stage_bytes) >> 4;
        int st = 0;
        uint32_t ph = 0, off = 0;
#pragma unroll 1
        for (int i = 0; i < k_count; i++) {
            if (!mbar_wait_warp<true>(&full_bar[st], ph, abort_flag, status, 0xA10 | (blockIdx.x << 12))) break;
            tc_fence_after_sync();
            if (elect_one()) {
                umma_chunk<1, AMN, BMN>(tmem_base, a0 + off, b0 + off, idesc, i != 0);
                if (i + p.stages < k_count) umma_commit(&empty_bar[st]);
                if (i == k_count - 1) umma_commit(&tfull_bar);
            }
            __syncwarp();
            off += stage16;
            if (++st == p.stages) { st = 0; ph ^= 1u; off = 0; }
        }
    } else {
        // ---- epilogue ----
        const int q = warp & 3, half = warp >> 2, m = q * 32 + lane;
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        const int out_bn = EPI == EPI_GATED ? p.BN / 2 : p.BN;
        bool ok = mbar_wait_warp<true>(&tfull_bar, 0u, abort_flag, status, 0xA20 | (blockIdx.x << 12));
        tc_fence_after_sync();
        if (SPLIT == 1) {
            // a lane finishes its own row, 8 outputs at a time
            const bool row_live = m < live && ok;
#pragma unroll 1
            for (int c = half * 16; c < out_bn; c += 32) {
                float v[16], u[16];
                tmem_ld16(taddr + c, v);
                if (EPI == EPI_GATED) tmem_ld16(taddr + out_bn + c, u);
#pragma unroll
                for (int g = 0; g < 2; g++)
                    if (row_live && n0 + c + g * 8 < p.N)
                        finish8<EPI, T>(p, group, m0 + m, n0 + c + g * 8, *reinterpret_cast<float(*)[8]>(v + g * 8), *reinterpret_cast<float(*)[8]>(u + g * 8));
                __syncwarp();
            }
        } else {
            const int dest = min(m / p.rows_per, SPLIT - 1), row = m - dest * p.rows_per;
            const uint32_t slab = static_cast<uint32_t>(p.rows_per * p.BN * 4);   // one rank's partial rows
            // (a row's 16-byte vectors are stored in an order that depends on the row: the lanes of a warp fall into different banks)
            const uint32_t dst = mapa(base + p.red_off + rank * slab + row * p.BN * 4, dest), dst_bar = mapa(smem_u32(&red_bar), dest);
            cluster_wait();   // every CTA of the cluster runs and its barrier expects these rows
#pragma unroll 1
            for (int c0 = half * 16; c0 < p.BN; c0 += 32) {
                float v[16];
                tmem_ld16(taddr + c0, v);
                if (m < live) {   // (sent whatever happened: the other CTAs wait for the bytes)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        st_async_v4(dst + ((static_cast<uint32_t>((c0 >> 2) + e) ^ (static_cast<uint32_t>(row) & 7u)) << 4), v[4 * e], v[4 * e + 1], v[4 * e + 2],
                                    v[4 * e + 3], dst_bar);
                }
                __syncwarp();
            }
            // All rows of this CTA are here.  It must not retire before that, whatever its own part came to, hence a limit above
            // the senders' and a flag of its own.
            ok = mbar_wait<true>(&red_bar, 0u, &red_abort_s, status, 0xA30 | (blockIdx.x << 12), 4 * kWaitLimitNs) && ok;
            const int my_rows = max(0, min(p.rows_per, live - rank * p.rows_per)), per_row = out_bn / 8;
            const uint8_t* red = sbase + p.red_off;
#pragma unroll 1
            for (int i = threadIdx.x; i < my_rows * per_row; i += 32 * kEpiWarps) {
                const int r = i / per_row, c = (i - r * per_row) * 8;
                if (!ok || n0 + c >= p.N) continue;
                float v[8] = {}, u[8] = {};
                auto sum = [&](int col, float (&s)[8]) {
                    const uint32_t at = static_cast<uint32_t>(r * p.BN * 4) + ((static_cast<uint32_t>(col >> 2) ^ (static_cast<uint32_t>(r) & 7u)) << 4);
#pragma unroll
                    for (int sp = 0; sp < SPLIT; sp++) {
                        const float4 x = *reinterpret_cast<const float4*>(red + sp * slab + at), y = *reinterpret_cast<const float4*>(red + sp * slab + (at ^ 16u));
                        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
                        s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
                    }
                };
                sum(c, v);
                if (EPI == EPI_GATED) sum(out_bn + c, u);
                finish8<EPI, T>(p, group, m0 + rank * p.rows_per + r, n0 + c, v, u);
            }
        }
        tc_fence_before_sync();
    }
    __syncwarp();
    if (SPLIT > 1 && warp >= kEpiWarps) cluster_wait();
    __syncthreads();
    if (warp == kMmaWarp) {
        if (abort_s) __nanosleep(20000);   // let copies in flight land before the CTA retires
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, kMaxBN);
    }
}

typedef void (*LatFn)(const LatParams);
template <typename T, int SPLIT>
LatFn pick_op(const DenseGemm& g) {
    if (g.gated) return dense_lat_kernel<T, false, false, EPI_GATED, SPLIT>;
    if (g.a_mn) return dense_lat_kernel<T, true, true, EPI_PLAIN, SPLIT>;
    if (g.b_mn) return dense_lat_kernel<T, false, true, EPI_PLAIN, SPLIT>;
    return dense_lat_kernel<T, false, false, EPI_LINEAR, SPLIT>;
}
template <typename T>
LatFn pick_lat(const DenseGemm& g, int split) {
    switch (split) {
        case 1: return pick_op<T, 1>(g);
        case 2: return pick_op<T, 2>(g);
        case 4: return pick_op<T, 4>(g);
        default: return pick_op<T, 8>(g);
    }
}

// The layout of a tile in shared memory: ring depth, and where the cluster's partial sums go.
bool lay_out(const DenseGemm& g, const DenseLatChoice& c, LatParams* p, size_t* smem) {
    p->BN = c.bn;
    p->rows = c.rows;
    p->a_bytes = g.a_mn ? 16384 : (c.rows + 7) / 8 * 1024;
    p->stage_bytes = p->a_bytes + c.bn * 128;
    p->chunks1 = static_cast<int>((g.K + 63) / 64);
    p->total = p->chunks1 * g.sources;
    p->share = (p->total + c.split - 1) / c.split;
    p->rows_per = (c.rows + c.split - 1) / c.split;
    if (c.split > 1 && (c.split - 1) * p->share >= p->total) return false;   // (a CTA without work)
    const int red = c.split > 1 ? c.split * p->rows_per * c.bn * 4 : 0;
    const int slack = 16384 - p->a_bytes;   // the tensor core reads 128 rows of A, behind the ring's last ones too: memory of this CTA all the same
    p->stages = std::min({kMaxStages, (kMaxDynSmem - 1024 - red - slack) / p->stage_bytes, p->share});
    if (p->stages < std::min(p->share, 3)) return false;
    p->red_off = p->stages * p->stage_bytes + slack;
    *smem = static_cast<size_t>(p->red_off) + red + 1024;
    if (c.split > 1) *smem = std::max<size_t>(*smem, kAloneSmem);
    return true;
}

}  // namespace

bool dense_lat_possible(const DenseGemm& g, const DenseLatChoice& c) {
    LatParams p;
    size_t smem;
    return lay_out(g, c, &p, &smem);
}

int launch_dense_lat(const DenseGemm& g, const DenseLatChoice& c, cudaStream_t s) {
    LatParams p;
    std::memset(&p, 0, sizeof(p));
    size_t smem = 0;
    if (!lay_out(g, c, &p, &smem)) return DLF_E_UNSUPPORTED;
    int rc = DLF_OK;
    for (int i = 0; i < 2 && rc == DLF_OK; i++) {
        const Mat &a = g.a[i], &b = g.b[i];
        if (a.p) rc = g.a_mn ? dense_map(&p.a[i], a, g.K, g.M, 64, 64) : dense_map(&p.a[i], a, g.M, g.K, p.a_bytes / 128, 64);
        if (b.p && rc == DLF_OK) rc = g.b_mn ? dense_map(&p.b[i], b, g.K, g.N, 64, 64) : dense_map(&p.b[i], b, g.N, g.K, g.gated ? c.bn / 2 : c.bn, 64);
    }
    if (rc) return rc;
    for (int i = 0; i < 3; i++) {
        p.o[i] = g.out[i];
        p.vec[i] = dense_rows16(g.out[i]);
    }
    p.res = g.res;
    p.res_vec = dense_rows16(g.res);
    p.bias[0] = g.bias[0]; p.bias[1] = g.bias[1];
    p.M = g.M; p.N = g.N;
    const int step = g.gated ? c.bn / 2 : c.bn;
    p.tiles_n = static_cast<int>((g.N + step - 1) / step);
    p.group_tiles = (g.M + c.rows - 1) / c.rows * p.tiles_n;
    p.act = g.act; p.groups = g.groups;
    const LatFn fn = g.dtype == DLF_BF16 ? pick_lat<__nv_bfloat16>(g, c.split) : pick_lat<__half>(g, c.split);
    rc = dense_smem_attr(reinterpret_cast<const void*>(fn), kMaxDynSmem);
    if (rc) return rc;
    const int grid = static_cast<int>(p.group_tiles * g.groups * c.split);
    const cudaError_t e = launch_kernel(fn, grid, kThreads, smem, s, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

int dense_lat_status(cudaStream_t s, int* code) { return dense_status_of(s, code); }

}  // namespace dlf
