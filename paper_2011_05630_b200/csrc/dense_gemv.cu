// Forward products of a few tokens (at most 16): what bounds them is the weights' way from memory, and a tile of the larger
// kernels would be mostly empty rows behind a longer way (shared memory, tensor memory, an exchange).  Here the weights go from
// memory straight into the registers of warp-level matrix instructions (16 weight rows x 8 tokens x 16 of K; their rate is
// of no account at 16 bytes of weights a lane for two of them): the order of K within an instruction is free as long as both operands
// have the same, so that a lane's 8 consecutive values of a row are its share of two instructions, and nothing is rearranged.
//
// A CTA has a run of weight rows for itself, all CTAs one of the same length, two CTAs to an SM: every SM streams until the end.  Its
// eight warps share K in blocks of consecutive values and meet in shared memory, in the order of the warps.  Rows may start anywhere:
// off the 16-byte boundaries a lane takes the two aligned pieces that hold its values and shifts them together.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_mem.cuh"
#include "ptx.cuh"

namespace cg = cooperative_groups;

namespace dlf {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

// Steps of 32 of K that a warp has on their way at a time: as many as 128 registers hold.
__host__ __device__ constexpr int steps_ahead(int nt, bool gated, bool any) {
    return gated ? (nt > 1 ? (any ? 2 : 3) : (any ? 3 : 4)) : nt > 1 ? 4 : (any ? 5 : 6);
}

struct GemvParams {
    Mat x, w[2], o[3], res;
    const float* bias[2];
    long long N;
    int M, K, act, rows, lg_ranks;   // weight rows of a CTA; CTAs of a cluster
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

// 8 values of which those below `from` and from `to` on are zeros.
__device__ __forceinline__ uint4 only(const uint4& q, int from, int to) {
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] &= (2 * i >= from && 2 * i < to ? 0xffffu : 0u) | (2 * i + 1 >= from && 2 * i + 1 < to ? 0xffff0000u : 0u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// A lane's 16 bytes from byte `shift` of its piece on: the rest of its piece and the start of the next one.  Four lanes have four pieces
// side by side; the fourth one's neighbour is the first one at the next step, `next`, or behind a block's last step a piece that
// the fourth lane has for itself.
__device__ __forceinline__ uint4 slide(const uint4& own, const uint4& next, bool last, int lane, uint32_t shift) {
    const int t = lane & 3, from = (lane & ~3) | ((t + 1) & 3);
    const uint4 send = t == 0 && !last ? next : own;
    uint4 b = make_uint4(__shfl_sync(0xffffffffu, send.x, from), __shfl_sync(0xffffffffu, send.y, from), __shfl_sync(0xffffffffu, send.z, from), __shfl_sync(0xffffffffu, send.w, from));
    if (last && t == 3) b = next;
    return shift16(own, b, shift);
}

// NT: runs of 8 tokens.  ANY: rows start anywhere, or end inside 16 bytes.  Launched in clusters, a cluster's CTAs share the K of the same rows.
//
// Rows off the 16-byte boundaries: eight rows further the distance to the boundary is the same, whatever the row length, so a CTA
// takes every eighth row.  Its weights go into the products as the pieces of 16 bytes that memory has, and the tokens' values are
// shifted to where these have their K: one realignment for all rows (all of the rows realigned instead: 4099 -> 11264, one token, 35.5 us
// against 24.1).  What lies beside a row in its first and last piece is masked out.
template <typename T, int NT, bool GATED, bool ANY>
__global__ void __launch_bounds__(kThreads, 2) dense_gemv_kernel(const __grid_constant__ GemvParams p) {
    constexpr int NW = GATED ? 2 : 1;   // weight matrices
    constexpr int D = steps_ahead(NT, GATED, ANY);
    constexpr int X = ANY ? D + 1 : D;   // (of the tokens one piece more)
    constexpr int kEvery = ANY ? 8 : 1;  // distance of a CTA's rows
    __shared__ float part_s[2][kWarps][NW * 16][8 * NT + 2];
    pdl_wait();
    pdl_launch_dependents();
    const int ranks = 1 << p.lg_ranks, rank = static_cast<int>(blockIdx.x) & (ranks - 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int group = static_cast<int>(blockIdx.x) >> p.lg_ranks, cls = group & (kEvery - 1);
    // this CTA's rows: cls + kEvery * i for i from first to end - 1
    const long long first = static_cast<long long>(group / kEvery) * p.rows, end = min(first + p.rows, (p.N - cls + kEvery - 1) / kEvery);
    const auto row_at = [&](const Mat& m, long long i) { return reinterpret_cast<uintptr_t>(m.p) + static_cast<uintptr_t>((cls + kEvery * i) * m.ld * 2); };
    const uint32_t shift = ANY ? static_cast<uint32_t>(row_at(p.w[0], 0) & 15) : 0u;   // bytes of a row's first piece in front of it
    const int pieces = static_cast<int>((shift + 2ll * p.K + 15) >> 4);                // of 16 bytes that hold values of a row
    // K goes round the cluster's warps in blocks of D steps (side by side: pieces of 64 bytes a row make the memory slower); the loads run
    // a block ahead of the products, into the next 16 rows too
    const int blocks = (((pieces + 3) / 4 + kWarps * D - 1) / (kWarps * D) + ranks - 1) >> p.lg_ranks;
    auto piece_of = [&](int block, int d) { return ((((block << p.lg_ranks) + rank) * kWarps + warp) * D + d) * 4 + t; };   // a lane's at step d of a block
    // tokens: the piece that holds the first value for piece 0 of the weights, and how far into it that value lies
    const char* x[NT];
    uint32_t x_shift[NT];
    int x_first[NT], x_end[NT];   // pieces, counted from that one, that hold values of the token
#pragma unroll
    for (int j = 0; j < NT; j++) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p.x.p) + static_cast<uintptr_t>(min(g + 8 * j, p.M - 1) * p.x.ld * 2);
        x_shift[j] = ANY ? static_cast<uint32_t>((at - shift) & 15) : 0u;
        x[j] = reinterpret_cast<const char*>(at - shift - x_shift[j]);
        const bool live = g + 8 * j < p.M;
        x_first[j] = ANY ? static_cast<int>((shift + x_shift[j]) >> 4) : 0;
        x_end[j] = live ? (ANY ? static_cast<int>((shift + x_shift[j] + 2ll * p.K + 15) >> 4) : pieces) : 0;
    }
    struct At {
        long long i0;
        const char* w[NW][2];
        int pieces[2];
        int block;
    };
    auto rows_of = [&](At& a) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const bool live = a.i0 + g + 8 * h < end;
            a.pieces[h] = live ? pieces : 0;
#pragma unroll
            for (int q = 0; q < NW; q++) a.w[q][h] = reinterpret_cast<const char*>(row_at(p.w[q], live ? a.i0 + g + 8 * h : first) - shift);
        }
    };
    uint4 wv[D][NW][2], xv[X][NT];
    auto fetch = [&](const At& a, int d) {
        // (behind a block's last step the fourth lane loads what would be the first one's next piece)
        const int at = piece_of(a.block, d) - (d == D ? 3 : 0);
        if (d < D) {
#pragma unroll
            for (int q = 0; q < NW; q++)
#pragma unroll
                for (int h = 0; h < 2; h++) wv[d < D ? d : 0][q][h] = ld16_if<true>(a.w[q][h] + static_cast<long long>(at) * 16, at < a.pieces[h]);
        }
#pragma unroll
        for (int j = 0; j < NT; j++) xv[d][j] = ld16_if<false>(x[j] + static_cast<long long>(at) * 16, (d < D || t == 3) && at >= x_first[j] && at < x_end[j]);
    };
    At ahead{first, {}, {}, 0};
    rows_of(ahead);
#pragma unroll
    for (int d = 0; d < X; d++) fetch(ahead, d);
    int buf = 0;
#pragma unroll 1
    for (long long i0 = first; i0 < end; i0 += 16, buf ^= 1) {
        float acc[NW][NT][4] = {};
#pragma unroll 1
        for (int block = 0; block < blocks; block++) {
            if (++ahead.block == blocks) {
                ahead.block = 0;
                ahead.i0 += 16;
                rows_of(ahead);   // (past the last row: nothing is live)
            }
#pragma unroll
            for (int d = 0; d < D; d++) {
                uint4 c[NT];
#pragma unroll
                for (int j = 0; j < NT; j++) c[j] = ANY ? slide(xv[d][j], xv[ANY ? d + 1 : d][j], d == D - 1, lane, x_shift[j]) : xv[d][j];
                if (ANY) {   // K of the lane's first value, and what is no value of the rows
                    const int k = piece_of(block, d) * 8 - static_cast<int>(shift >> 1);
                    if (k < 0 || k + 8 > p.K) {
#pragma unroll
                        for (int j = 0; j < NT; j++) c[j] = only(c[j], -k, p.K - k);
#pragma unroll
                        for (int q = 0; q < NW; q++)
#pragma unroll
                            for (int h = 0; h < 2; h++) wv[d][q][h] = only(wv[d][q][h], -k, p.K - k);
                    }
                }
#pragma unroll
                for (int q = 0; q < NW; q++) {
                    const uint4 &a = wv[d][q][0], &b = wv[d][q][1];
#pragma unroll
                    for (int j = 0; j < NT; j++) {
                        mma16816<T>(acc[q][j], a.x, b.x, a.y, b.y, c[j].x, c[j].y);
                        mma16816<T>(acc[q][j], a.z, b.z, a.w, b.w, c[j].z, c[j].w);
                    }
                }
                fetch(ahead, d);
            }
            if (ANY) fetch(ahead, X - 1);
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
        const long long n = cls + kEvery * (i0 + r);
        const bool live = m < p.M && m < 8 * NT && i0 + r < end;
        float z = 0.0f, u = 0.0f;
        auto total = [&](int row) {   // (in the warps' order)
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < kWarps; i++) v += part_s[buf][i][row][m];
            return v;
        };
        if (live) {
            z = total(r);
            if (GATED) u = total(GATED ? 16 + r : 0);
        }
        if (ranks > 1) {   // in the ranks' order; the first one finishes
            cg::cluster_group cluster = cg::this_cluster();
            if (live) {
                part_s[buf][0][r][m] = z;   // (a thread's own column of its own row)
                if (GATED) part_s[buf][0][GATED ? 16 + r : 0][m] = u;
            }
            cluster.sync();
            if (live && rank == 0)
                for (int i = 1; i < ranks; i++) {
                    z += *cluster.map_shared_rank(&part_s[buf][0][r][m], i);
                    if (GATED) u += *cluster.map_shared_rank(&part_s[buf][0][GATED ? 16 + r : 0][m], i);
                }
            cluster.sync();   // no CTA goes on while its sums are still read
        }
        if (live && rank == 0) {
            auto put = [&](const Mat& o, float v) { static_cast<T*>(const_cast<void*>(o.p))[m * o.ld + n] = from_f32<T>(v); };
            if (p.bias[0]) z += ld_map(p.bias[0] + n);
            if (GATED) {
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

// (a gated block's two matrices have to lie the same way to the 16-byte boundaries)
bool dense_gemv_takes(const DenseGemm& g) {
    if (g.M > 16) return false;
    auto same = [](const Mat& a, const Mat& b) { return ((reinterpret_cast<uintptr_t>(a.p) ^ reinterpret_cast<uintptr_t>(b.p)) & 15) == 0 && (a.ld - b.ld) % 8 == 0; };
    return !g.gated || same(g.b[0], g.b[1]);
}

DenseGemvLayout dense_gemv_layout(const DenseGemm& g, int sms) {
    DenseGemvLayout l;
    l.any = g.K % 8 != 0 || !dense_rows16(g.a[0]) || !dense_rows16(g.b[0]) || !dense_rows16(g.b[1]);
    const int64_t classes = l.any ? 8 : 1, per_class = (g.N + classes - 1) / classes;
    l.rows = static_cast<int>(std::max<int64_t>(8, (g.N + 2 * sms - 1) / (2 * sms)));
    l.groups = classes * ((per_class + l.rows - 1) / l.rows);
    // Few rows: their K is shared out over the CTAs of a cluster where there is room for them and enough work: a block of a warp's steps
    // takes about 0.8 us, meeting in a cluster 1.7 (10094 -> 624, gated, one token: 16 -> 12 us; 2048 -> 1000: 3.4 -> 4.3, not done).
    const int64_t block = kWarps * 32 * steps_ahead(g.M > 8 ? 2 : 1, g.gated, l.any);
    l.blocks = (g.K + block - 1) / block;
    l.lg_ranks = 0;
    double least = 0.8 * static_cast<double>(l.blocks);
    for (int lg = 1; lg <= 3 && (l.groups << lg) <= 2 * sms; lg++) {
        const double us = 0.8 * static_cast<double>((l.blocks + (1 << lg) - 1) >> lg) + 1.7;
        if (us < least) {
            least = us;
            l.lg_ranks = lg;
        }
    }
    return l;
}

int launch_dense_gemv(const DenseGemm& g, int sms, cudaStream_t s) {
    const DenseGemvLayout l = dense_gemv_layout(g, sms);
    const bool any = l.any;
    const int64_t groups = l.groups;
    GemvParams p{};
    p.x = g.a[0];
    for (int i = 0; i < 2; i++) { p.w[i] = g.b[i]; p.bias[i] = g.bias[i]; }
    for (int i = 0; i < 3; i++) p.o[i] = g.out[i];
    p.res = g.res;
    p.N = g.N; p.M = static_cast<int>(g.M); p.K = static_cast<int>(g.K); p.act = g.act;
    p.rows = l.rows;
    p.lg_ranks = l.lg_ranks;
    const int ranks = 1 << p.lg_ranks;
    const bool bf = g.dtype == DLF_BF16;
    const GemvFn fn = g.M > 8 ? (bf ? pick_gemv<__nv_bfloat16, 2>(g.gated, any) : pick_gemv<__half, 2>(g.gated, any))
                              : (bf ? pick_gemv<__nv_bfloat16, 1>(g.gated, any) : pick_gemv<__half, 1>(g.gated, any));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(groups * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (g_use_pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (ranks > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = static_cast<unsigned>(ranks);
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        n++;
    }
    cfg.attrs = attr;
    cfg.numAttrs = static_cast<unsigned>(n);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

}  // namespace dlf
