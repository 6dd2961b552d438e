// Host side of the dense operators (dlf_linear*, dlf_gated*), and the pass that takes gradients back through an activation.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <type_traits>

#include "dense.h"
#include "dense_math.cuh"
#include "dense_mem.cuh"
#include "ptx.cuh"

namespace cg = cooperative_groups;

namespace dlf {

namespace {

// ---- gradients behind an activation ----------------------------------------------------------------------------------------
// Bound by memory: 2 or 3 matrices are read, 1 or 2 written, once each.  A CTA owns 64 columns (128 bytes of a row: whole lines; 16 where
// a narrow matrix would leave SMs without work) and walks rows, so that a column's sum stays in one thread's registers; kGradSplit CTAs
// share the rows of a strip as a cluster and their column sums meet in distributed shared memory, added up in the order of the ranks:
// the same bits every time, no atomics and no second kernel.
constexpr int kGradCols = 64, kNarrowCols = 16, kGradThreads = 128, kGradSplit = 8;

// V values of a row, as they lie in memory: 8 on a 16-byte boundary (they come through shared memory), or 2 anywhere, n of which exist.
template <typename T, int V>
struct Run;
template <typename T>
struct Run<T, 8> {
    uint4 q;
    __device__ __forceinline__ float2 get2(int i) const { return unpack2<T>(i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w); }
    __device__ __forceinline__ void set2(int i, float2 f) { (i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w) = pack2<T>(f.x, f.y); }
    __device__ __forceinline__ void store(const Mat& m, int64_t row, int64_t col, int) const {
        if (m.p) *reinterpret_cast<uint4*>(static_cast<T*>(const_cast<void*>(m.p)) + row * m.ld + col) = q;
    }
};
template <typename T>
struct Run<T, 2> {
    uint32_t q;
    __device__ __forceinline__ void load(const Mat& m, int64_t row, int64_t col, int n) {
        const unsigned short* p = static_cast<const unsigned short*>(m.p) + row * m.ld + col;
        const uint32_t lo = n > 0 ? ld_map(p) : 0u, hi = n > 1 ? ld_map(p + 1) : 0u;
        q = lo | hi << 16;
    }
    __device__ __forceinline__ float2 get2(int) const { return unpack2<T>(q); }
    __device__ __forceinline__ void set2(int, float2 f) { q = pack2<T>(f.x, f.y); }
    __device__ __forceinline__ void store(const Mat& m, int64_t row, int64_t col, int n) const {
        if (!m.p) return;
        unsigned short* p = static_cast<unsigned short*>(const_cast<void*>(m.p)) + row * m.ld + col;
        p[0] = static_cast<unsigned short>(q);
        if (n > 1) p[1] = static_cast<unsigned short>(q >> 16);
    }
};

// 16 bytes to shared memory, counted by the thread's groups of copies.
__device__ __forceinline__ void copy16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

template <typename T, int V, bool GATED, int ACT, bool WIDE>
__global__ void __cluster_dims__(kGradSplit, 1, 1) __launch_bounds__(kGradThreads, GATED ? 5 : 7) dense_grad_kernel(const __grid_constant__ DenseGrad g) {
    constexpr int kParts = kGradThreads / 32;   // partial sums of a column: a warp's
    constexpr int width = WIDE ? kGradCols : kNarrowCols, tx_n = width / V;   // columns of the strip, threads of a row
    __shared__ float red[GATED ? 2 : 1][kParts][kGradCols];
    pdl_wait();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank());
    const int64_t strip = blockIdx.x / kGradSplit;
    const int tx = threadIdx.x & (tx_n - 1), ty = threadIdx.x / tx_n;
    const int64_t col = strip * width + tx * V;
    const int n = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(V), g.N - col)));   // (with V == 8 the columns are a multiple of 8)
    constexpr int VP = V / 2;   // pairs of values
    float2 s0[VP] = {}, s1[VP] = {};
    // rows are dealt out round by round, so that the CTAs of a strip are never far apart
    constexpr int64_t rows_at_once = kGradThreads / tx_n, kStep = rows_at_once * kGradSplit;
    const int64_t first = rank * rows_at_once + ty;
    constexpr bool kWithZ = GATED || ACT != DLF_ACT_NONE;
    auto work = [&](int64_t row, const Run<T, V>& dy, const Run<T, V>& z, const Run<T, V>& u) {
        Run<T, V> d, e;
#pragma unroll
        for (int i = 0; i < VP; i++) {
            constexpr bool kCorner = ACT == DLF_ACT_RELU || ACT == DLF_ACT_RELU6;   // (its slope chooses, last)
            float2 value, slope;
            float2 t = dy.get2(i);
            act_grad2<ACT>(kWithZ ? z.get2(i) : t, &value, &slope);
            if (GATED) {
                const float2 q = mul2(t, value);
                s1[i] = add2(s1[i], q);
                e.set2(i, q);
                if (kCorner) t = mul2(t, u.get2(i));
                else slope = mul2(slope, u.get2(i));
            }
            const float2 q = behind2<ACT>(t, slope);
            s0[i] = add2(s0[i], q);
            d.set2(i, q);
        }
        d.store(g.d0, row, col, n);
        if (GATED) e.store(g.d1, row, col, n);
        else d.store(g.d0c, row, col, n);
    };
    if constexpr (V == 8) {
        // a thread's next rows come into places of its own in shared memory (nobody else's: nothing to meet for), kAhead - 1 rows ahead
        // of the one worked on: 16 KB of places for a CTA, 24 gated, without a register for them.  Against two rows ahead in registers,
        // 4096 x 5632: GELU with its gradient written 32.5 -> 29.4 us (30.9 with normal2 as it is now), SILU gated with the sums alone
        // 38.3 -> 25.5; six places 30.1 and 28.7.
        constexpr int kAhead = 4, kArrays = GATED ? 3 : kWithZ ? 2 : 1;
        __shared__ uint4 ring[kAhead][kArrays][kGradThreads];
        auto fetch = [&](int64_t row, int slot) {
            if (n > 0 && row < g.M) {
                copy16(&ring[slot][0][threadIdx.x], static_cast<const T*>(g.dy.p) + row * g.dy.ld + col);
                if (kWithZ) copy16(&ring[slot][kWithZ ? 1 : 0][threadIdx.x], static_cast<const T*>(g.z.p) + row * g.z.ld + col);
                if (GATED) copy16(&ring[slot][GATED ? 2 : 0][threadIdx.x], static_cast<const T*>(g.u.p) + row * g.u.ld + col);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < kAhead - 1; i++) fetch(first + i * kStep, i);
        int slot = 0;
        if (n > 0)
#pragma unroll 1
            for (int64_t row = first; row < g.M; row += kStep) {
                fetch(row + (kAhead - 1) * kStep, slot == 0 ? kAhead - 1 : slot - 1);
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
                Run<T, V> dy, z, u;
                dy.q = ring[slot][0][threadIdx.x];
                if (kWithZ) z.q = ring[slot][kWithZ ? 1 : 0][threadIdx.x];
                if (GATED) u.q = ring[slot][GATED ? 2 : 0][threadIdx.x];
                work(row, dy, z, u);
                if (++slot == kAhead) slot = 0;
            }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    } else {
        constexpr int kRows = 4;   // rows of a thread on their way at a time, twice: these and the next ones
        Run<T, V> dy[2][kRows], z[2][kRows], u[2][GATED ? kRows : 1];
        auto fetch = [&](int b, int64_t row0) {
#pragma unroll
            for (int r = 0; r < kRows; r++) {
                const int64_t row = row0 + r * kStep;
                const int here = row < g.M ? n : 0;
                dy[b][r].load(g.dy, row, col, here);
                if (kWithZ) z[b][r].load(g.z, row, col, here);
                if (GATED) u[b][GATED ? r : 0].load(g.u, row, col, here);
            }
        };
        auto turn = [&](int b, int64_t row0) {
#pragma unroll
            for (int r = 0; r < kRows; r++) {
                if (row0 + r * kStep >= g.M) break;
                work(row0 + r * kStep, dy[b][r], z[b][r], u[b][GATED ? r : 0]);
            }
        };
        if (n > 0) {
            int64_t row0 = first;
            fetch(0, row0);
#pragma unroll 1
            while (row0 < g.M) {
                fetch(1, row0 + kRows * kStep);
                turn(0, row0);
                row0 += kRows * kStep;
                if (row0 >= g.M) break;
                fetch(0, row0 + kRows * kStep);
                turn(1, row0);
                row0 += kRows * kStep;
            }
        }
    }
    if (!g.db0 && !g.db1) return;   // (the same for every thread of the cluster)
    // the rows of a warp
    auto meet = [&](float2 v) {
#pragma unroll
        for (int d = tx_n; d < 32; d <<= 1) v = add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, d), __shfl_xor_sync(0xffffffffu, v.y, d)));
        return v;
    };
#pragma unroll
    for (int i = 0; i < VP; i++) {
        s0[i] = meet(s0[i]);
        if (GATED) s1[i] = meet(s1[i]);
    }
    if (static_cast<int>(threadIdx.x & 31) < tx_n) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            red[0][threadIdx.x / 32][tx * V + i] = i & 1 ? s0[i / 2].y : s0[i / 2].x;
            if (GATED) red[GATED ? 1 : 0][threadIdx.x / 32][tx * V + i] = i & 1 ? s1[i / 2].y : s1[i / 2].x;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (GATED ? 2 : 1) * kGradCols; i += kGradThreads) {
        const int which = i / kGradCols, c = i % kGradCols;
        if (c >= width) continue;
        float s = 0.0f;
#pragma unroll
        for (int y = 0; y < kParts; y++) s += red[which][y][c];
        red[which][0][c] = s;
    }
    cluster.sync();
    if (rank == 0)
        for (int i = threadIdx.x; i < (GATED ? 2 : 1) * kGradCols; i += kGradThreads) {
            const int which = i / kGradCols, c = i % kGradCols;
            float s = 0.0f;
            for (int r = 0; r < kGradSplit; r++) s += *cluster.map_shared_rank(&red[which][0][c], r);
            float* db = which ? g.db1 : g.db0;
            if (db && c < width && strip * width + c < g.N) db[strip * width + c] = s;
        }
    cluster.sync();   // no CTA leaves while its sums are still read
}

typedef void (*GradFn)(const DenseGrad);
template <typename T, int V, bool GATED, bool WIDE>
GradFn pick_grad_act(int act) {
    switch (act) {
        case DLF_ACT_RELU: return dense_grad_kernel<T, V, GATED, DLF_ACT_RELU, WIDE>;
        case DLF_ACT_RELU6: return dense_grad_kernel<T, V, GATED, DLF_ACT_RELU6, WIDE>;
        case DLF_ACT_GELU: return dense_grad_kernel<T, V, GATED, DLF_ACT_GELU, WIDE>;
        case DLF_ACT_GELU_TANH: return dense_grad_kernel<T, V, GATED, DLF_ACT_GELU_TANH, WIDE>;
        case DLF_ACT_SILU: return dense_grad_kernel<T, V, GATED, DLF_ACT_SILU, WIDE>;
        default: return dense_grad_kernel<T, V, GATED, DLF_ACT_NONE, WIDE>;
    }
}
template <typename T, int V>
GradFn pick_grad(bool gated, bool wide, int act) {
    if (gated) return wide ? pick_grad_act<T, V, true, true>(act) : pick_grad_act<T, V, true, false>(act);
    return wide ? pick_grad_act<T, V, false, true>(act) : pick_grad_act<T, V, false, false>(act);
}

// How the pass runs: 8 values at a time or 2 (see Run), wide strips or narrow ones, CTAs.
struct GradLayout {
    bool v8, wide;
    int grid;
};
GradLayout grad_layout(const DenseGrad& g, int sms) {
    auto vec = [](const Mat& m) { return !m.p || (aligned(16, m.p) && m.ld % 8 == 0); };
    auto strips = [&](int cols) { return (g.N + cols - 1) / cols * kGradSplit; };
    GradLayout l;
    l.v8 = g.N % 8 == 0 && vec(g.dy) && vec(g.z) && vec(g.u) && vec(g.d0) && vec(g.d1) && vec(g.d0c);
    // Strips of 64 columns where they give every SM two CTAs or the rows are few, else of 16.  GELU with its gradient written, wide -> narrow:
    // 1000 rows of 128 3.6 -> 2.6 us, 6428 of 128 12.0 -> 4.7, 20000 of 33 127 -> 36; but 512 of 1024 3.3 -> 4.1.  (Between the two the rule is up to
    // 2 us off, 2048 of 2048 7.8 -> 9.6, and below 1000 rows more where they are off the boundaries: 900 of 130 7.8 -> 3.6.)
    l.wide = strips(kGradCols) >= 2 * sms || g.M < 1000;
    l.grid = static_cast<int>(strips(l.wide ? kGradCols : kNarrowCols));   // (at most 2^29)
    return l;
}

// ---- rows onto 16-byte boundaries --------------------------------------------------------------------------------------------
// For operands whose rows start anywhere: the tensor-core kernels load tiles by TMA, which takes 16-byte boundaries only.  A copy costs
// 4 bytes a value once, where a product reads the operand's tiles many times.  All of a call's operands in one launch; two aligned pieces
// of 16 bytes are read for each piece written.
struct PackParams {
    DensePack job[kMaxPacks];
    int64_t first[kMaxPacks + 1];   // pieces of 16 bytes before a job's
    int n;
};
template <typename I>   // (what counts the pieces: a division in 64 bits costs several times the copy)
__global__ void __launch_bounds__(256) dense_pack_kernel(const __grid_constant__ PackParams p) {
    constexpr int kItems = 4;       // pieces of a thread on their way at a time
    pdl_wait();
    pdl_launch_dependents();
    for (int q = 0; q < p.n; q++) {
        const DensePack& d = p.job[q];
        const I total = static_cast<I>(p.first[q + 1] - p.first[q]), per_row = static_cast<I>((d.cols + 7) / 8), threads = static_cast<I>(gridDim.x) * 256;
        for (I i0 = static_cast<I>(blockIdx.x) * 256 + threadIdx.x; i0 < total; i0 += kItems * threads) {
            uint4 v[kItems], *to[kItems];
#pragma unroll
            for (int e = 0; e < kItems; e++) {
                const I i = i0 + e * threads, row = i / per_row, c = (i - row * per_row) * 8;
                const bool in = i < total;
                to[e] = reinterpret_cast<uint4*>(static_cast<unsigned short*>(const_cast<void*>(d.to.p)) + static_cast<int64_t>(row) * d.to.ld + c);
                v[e] = load8_any(static_cast<const unsigned short*>(d.from.p) + static_cast<int64_t>(row) * d.from.ld + c,
                                 in ? static_cast<int>(min(static_cast<int64_t>(8), d.cols - static_cast<int64_t>(c))) : 0);
            }
#pragma unroll
            for (int e = 0; e < kItems; e++)
                if (i0 + e * threads < total) *to[e] = v[e];
        }
    }
}

// ---- arguments -------------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxDim = 1ll << 30, kMaxLd = 1ll << 36;

int check_sizes(int dtype, int act, int64_t m, int64_t k, int64_t n) {
    if (dtype != DLF_F16 && dtype != DLF_BF16) return DLF_E_INVALID_ARG;
    if (act < DLF_ACT_NONE || act > DLF_ACT_SILU) return DLF_E_INVALID_ARG;
    if (m < 0 || k < 1 || n < 1 || m > kMaxDim || k > kMaxDim || n > kMaxDim) return DLF_E_SHAPE;
    return DLF_OK;
}

// Collects a call's matrices: the first thing that is wrong with one of them, and their normalised form (the row length of a
// matrix of one row is nobody's business).
struct Mats {
    int rc = DLF_OK;
    Mat operator()(const void* p, int64_t rows, int64_t cols, int64_t ld, bool required) {
        if (!p) {
            if (required && rc == DLF_OK) rc = DLF_E_INVALID_ARG;
            return Mat{nullptr, 0};
        }
        if (rc == DLF_OK && !aligned(2, p)) rc = DLF_E_INVALID_ARG;
        if (rows <= 1) ld = (cols + 7) / 8 * 8;
        if (rc == DLF_OK && (ld < cols || ld > kMaxLd)) rc = DLF_E_SHAPE;
        return Mat{p, ld};
    }
    const float* vec(const float* p) {
        if (rc == DLF_OK && !aligned(4, p)) rc = DLF_E_INVALID_ARG;
        return p;
    }
};

// True if an output is an input or another output (the pairs that may be the same are left out by the caller).
bool shared(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
    for (auto o = outputs.begin(); o != outputs.end(); o++) {
        if (!*o) continue;
        for (auto q = outputs.begin(); q != o; q++)
            if (*q == *o) return true;
        for (const void* i : inputs)
            if (i == *o) return true;
    }
    return false;
}

// Hands out 256-byte aligned pieces of a workspace; with a null base it only counts.
struct Carver {
    unsigned char* base;
    size_t used = 0;
    void* operator()(size_t bytes) {
        void* p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
    // (rows on 128-byte lines: a tile's row of 128 bytes then is one of them)
    Mat matrix(int64_t rows, int64_t cols) {
        const int64_t ld = (cols + 63) / 64 * 64;
        return Mat{(*this)(static_cast<size_t>(rows) * ld * 2), ld};
    }
};

int check_workspace(const void* ws, size_t bytes, size_t need) {
    if (need == 0) return DLF_OK;
    return ws && bytes >= need && aligned(256, ws) ? DLF_OK : DLF_E_WORKSPACE;
}

int zero_matrix(const Mat& m, int64_t rows, int64_t cols, cudaStream_t s) {
    if (!m.p) return DLF_OK;
    const cudaError_t e = cudaMemset2DAsync(const_cast<void*>(m.p), static_cast<size_t>(m.ld) * 2, 0, static_cast<size_t>(cols) * 2, static_cast<size_t>(rows), s);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}
int zero_vec(float* p, int64_t n, cudaStream_t s) {
    if (!p) return DLF_OK;
    const cudaError_t e = cudaMemsetAsync(p, 0, static_cast<size_t>(n) * 4, s);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

// ---- which kernel --------------------------------------------------------------------------------------------------------------
// Microseconds among other kernels, for each kernel and layout that can run a product: fitted to 4000 measured times of 468 products
// (forward, gated and both gradients, 5 to 2048 tokens, widths from 256 to 11264; root mean square of the logarithm 0.11 and
// 0.09).  What is chosen by it takes 2.0 % longer than each product's best in the geometric mean, the best of the pairs alone 33 %, the
// best of the clusters alone (where they can run at all) 10 %.
double gemm_bytes(const DenseGemm& g) {
    const double m = static_cast<double>(g.M), n = static_cast<double>(g.N), k = static_cast<double>(g.K);
    return 2.0 * (m * k * std::max(g.sources, g.groups) + n * k * (g.gated ? 2 : g.sources) + m * n * g.groups);
}
// The longer of two times that overlap, a little more where they are near one another.
double longer(double a, double b) { return std::sqrt(std::sqrt(a * a * a * a + b * b * b * b)); }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// 1 if rows start off the 128-byte lines: a tile's row of 128 bytes then takes two of them (777 x 1000 x 1001: 8.9 us with x's rows 1024
// values apart, 10.0 with 1000).
double off_lines(const Mat (&m)[2]) { return (m[0].ld | (m[1].p ? m[1].ld : 0)) % 64 != 0 ? 1.0 : 0.0; }

double lat_cost(const DenseGemm* g, int n, int sms, DenseLatChoice* best) {
    double least = -1.0;
    DenseLatChoice c{};
    for (c.bn = 64; c.bn <= 128; c.bn += g[0].b_mn ? 64 : 32)   // (an operand across K comes in boxes of 64)
        for (c.split = 1; c.split <= 8; c.split *= 2) {
            int64_t ctas[2] = {}, all = 0;
            for (int j = 0; j < n; j++) all += ctas[j] = ceil_div(g[j].M, 128) * ceil_div(g[j].N, g[j].gated ? c.bn / 2 : c.bn) * g[j].groups * c.split;
            if (all > (1 << 20)) break;
            c.deep = all <= sms;
            int rows[2], stages[2];
            bool two = true, possible = true;
            for (int j = 0; j < n && possible; j++) {
                bool fits = false;
                possible = dense_lat_possible(g[j], c, &rows[j], &stages[j], &fits);
                two = two && fits;
            }
            if (!possible) continue;
            // clusters find fewer places than single CTAs: 148, 132 and 120 CTAs of clusters of 2, 4 and 8 on 148 SMs
            const double slots = sms * (c.split == 1 ? (two ? 2.0 : 1.0) : c.split == 2 ? 1.0 : c.split == 4 ? 132.0 / 148 : 120.0 / 148);
            const double waves = std::ceil(static_cast<double>(all) / slots);
            const double busy = std::min(two ? 2.0 : 1.0, std::max(1.0, static_cast<double>(all) / sms));   // CTAs of an SM at a time
            double longest = 0.0, mean = 0.0, bytes = 0.0;
            for (int j = 0; j < n; j++) {
                const double share = static_cast<double>(ceil_div(ceil_div(g[j].K, 64) * g[j].sources, c.split));
                const double stage = (g[j].a_mn ? 16384 : (rows[j] + 7) / 8 * 1024) * (1.0 + 0.54 * off_lines(g[j].a)) + c.bn * 128 * (1.0 + 0.54 * off_lines(g[j].b));
                // a chunk: its matrix instructions and what lies between two runs, its bytes at an SM's rate, a round trip shared by the ring
                double chunk = std::max(0.141 + 0.0004 * c.bn, stage * busy / 126e3);
                if (stages[j] < share) chunk = std::max(chunk, 1.17 / stages[j]);
                const double one = 2.61 + share * chunk + (c.split > 1 ? 1.1 + 2.5e-4 * rows[j] * c.bn : 8.5e-5 * rows[j] * c.bn);
                longest = std::max(longest, one);
                mean += one * static_cast<double>(ctas[j]) / static_cast<double>(all);
                bytes += gemm_bytes(g[j]);
            }
            const double us = longer(longest + (waves - 1.0) * (mean - (two ? 0.54 : 0.0)), 2.61 + bytes / 4.84e6);
            if (least < 0 || us < least) {
                least = us;
                *best = c;
            }
        }
    return least;
}
double pair_cost(const DenseGemm* g, int n, int sms, int bn) {
    double off = 0.0, bytes = 0.0;
    for (int j = 0; j < n; j++) {
        off += (off_lines(g[j].a) + off_lines(g[j].b)) / n;
        bytes += gemm_bytes(g[j]);
    }
    const double chunks = dense_pair_share(g, n, bn, sms).chunks;
    if (chunks < 0) return -1.0;
    // (two products side by side share less of what they load, as measured over 112 pairs of gradients)
    const double apart = n > 1 ? (bn == 256 ? 1.05 : 1.15) : 1.0;
    return apart * longer(1.56 + chunks * (bn == 256 ? 0.308 : 0.272) * (1.0 + 0.05 * off) + (bn == 256 ? 2.43 : 1.83), 1.56 + bytes / 5.79e6);
}

// The fastest launch of these products together, by the estimates.
struct GemmPlan {
    double us;
    bool lat;
    int bn;
    DenseLatChoice c;
};
GemmPlan plan_gemm(const DenseGemm* g, int n, int sms) {
    GemmPlan best{pair_cost(g, n, sms, 256), false, 256, {}};
    const double narrow = g[0].gated ? -1.0 : pair_cost(g, n, sms, 128);
    if (narrow >= 0 && (best.us < 0 || narrow < best.us)) best = GemmPlan{narrow, false, 128, {}};
    DenseLatChoice c{};
    const double lat = lat_cost(g, n, sms, &c);
    if (lat >= 0 && (best.us < 0 || lat < best.us)) best = GemmPlan{lat, true, 0, c};
    return best;
}
// What a call would do, asked for without doing it: the workspace that it wants, or the kernels that it launches, in their order.
struct Ask {
    size_t* workspace;
    char* text;   // (null: the workspace is asked for)
    size_t bytes, used;
    int sms;
    int say(const char* format, ...) {
        const char* const between = used ? "; " : "";
        if (used < bytes) used += static_cast<size_t>(std::snprintf(text + used, bytes - used, "%s", between));
        va_list args;
        va_start(args, format);
        if (used < bytes) used += static_cast<size_t>(std::max(0, std::vsnprintf(text + used, bytes - used, format, args)));
        va_end(args);
        return DLF_OK;
    }
};

// A call's launches - or, asked for, their names and what the host chose about them.
struct Steps {
    cudaStream_t s;
    Ask* ask;
    int sms = 0;
    int begin() {
        if (ask) sms = ask->sms;
        return sms > 0 ? DLF_OK : query_sms(&sms);
    }
    int pack(const DensePack* jobs, int n) {
        if (n == 0) return DLF_OK;
        return ask ? ask->say("dense_pack(matrices=%d)", n) : launch_dense_pack(jobs, n, sms, s);
    }
    int grad(const DenseGrad& g) {
        if (!ask) return launch_dense_grad(g, sms, s);
        const GradLayout l = grad_layout(g, sms);
        return ask->say("dense_grad(rows=%s columns=%d)", l.v8 ? "aligned" : "anywhere", l.wide ? kGradCols : kNarrowCols);
    }
    int gemv(const DenseGemm& g) {
        if (!ask) return launch_dense_gemv(g, sms, s);
        const DenseGemvLayout l = dense_gemv_layout(g, sms);
        return ask->say("dense_gemv(tokens=%d rows=%s blocks=%d split=%d)", g.M > 8 ? 16 : 8, l.any ? "anywhere" : "aligned", static_cast<int>(l.blocks), 1 << l.lg_ranks);
    }
    int plan(const GemmPlan& p, const DenseGemm* g, int n) {
        if (p.us < 0) return DLF_E_UNSUPPORTED;
        if (!ask) return p.lat ? launch_dense_lat(g, n, p.c, s) : launch_dense_pair(g, n, p.bn, sms, s);
        auto whole = [&](const DenseGemm& q, const Mat& m) { return !m.p || (dense_rows16(m) && q.N % 8 == 0); };   // (rows leave or come in pieces of 16 bytes)
        bool all = true;
        for (int j = 0; j < n; j++)
            for (const Mat& m : g[j].out) all = all && whole(g[j], m);
        const char* const out = all ? "aligned" : "anywhere";
        const char* const res = !g[0].res.p ? "none" : whole(g[0], g[0].res) ? "aligned" : "anywhere";
        if (p.lat) return ask->say("dense_lat(products=%d columns=%d split=%d sources=%d out=%s residual=%s)", n, p.c.bn, p.c.split, g[0].sources, out, res);
        const DensePairShare t = dense_pair_share(g, n, p.bn, sms);
        return ask->say("dense_pair(products=%d columns=%d sources=%d groups=%d pairs=%d rest=%d few=%d many=%d out=%s residual=%s)", n, p.bn, g[0].sources,
                        g[n - 1].groups, t.pairs, t.rest, t.few, t.many, out, res);
    }
    int gemm(const DenseGemm& g) { return plan(plan_gemm(&g, 1, sms), &g, 1); }
    // The gradients of an input and of weights: as one launch where its tiles fill the chip better than two launches' (4096 x 4096 x 4096:
    // 186 -> 171 us; 200 x 2048 x 1000, with the bias's: 15.1 -> 11.2), else one after the other.
    int grads(DenseGemm* g, int n) {
        if (n == 0) return DLF_OK;
        if (n == 1) return gemm(g[0]);
        if (g[0].K * g[0].sources < g[1].K * g[1].sources) std::swap(g[0], g[1]);   // the longer tiles first, the shorter ones fill up
        const GemmPlan one[2] = {plan_gemm(&g[0], 1, sms), plan_gemm(&g[1], 1, sms)}, both = plan_gemm(g, 2, sms);
        if (both.us >= 0 && both.us < one[0].us + one[1].us) return plan(both, g, 2);
        const int rc = plan(one[0], &g[0], 1);
        return rc ? rc : plan(one[1], &g[1], 1);
    }
    int zero(const Mat& m, int64_t rows, int64_t cols) { return ask ? DLF_OK : zero_matrix(m, rows, cols, s); }
    int zero(float* p, int64_t n) { return ask ? DLF_OK : zero_vec(p, n, s); }
};

// An operand as the products read it: itself, or a copy in the workspace (one of `jobs`).
struct Operands {
    Carver& carve;
    DensePack jobs[kMaxPacks];
    int n = 0;
    Mat operator()(const Mat& m, int64_t rows, int64_t cols) {
        if (!m.p || dense_rows16(m)) return m;
        const Mat to = carve.matrix(rows, cols);
        jobs[n++] = DensePack{rows, cols, m, to};
        return to;
    }
};

// ---- the four operators; with `ask` they only say what they would do -----------------------------------------------------------
// (Asked for the kernels: a workspace to lay out, at an address that nothing is read from.)
unsigned char* base_of(void* ws, const Ask* ask) { return ask && ask->text ? reinterpret_cast<unsigned char*>(256) : static_cast<unsigned char*>(ws); }
// What a call wants, once that is known; true if nothing else was asked for.
bool only_workspace(const Ask* ask, size_t bytes) {
    if (!ask || ask->text) return false;
    *ask->workspace = bytes;
    return true;
}
int ready(const Ask* ask, const void* ws, size_t bytes, size_t need, Steps* steps) {
    const int rc = ask ? DLF_OK : check_workspace(ws, bytes, need);
    return rc ? rc : steps->begin();
}

int linear(const dlf_linear_args* a, void* ws, size_t ws_bytes, cudaStream_t s, Ask* ask) {
    if (!a) return DLF_E_INVALID_ARG;
    int rc = check_sizes(a->dtype, a->act, a->m, a->k, a->n);
    if (rc) return rc;
    Mats mat;
    DenseGemm g{};
    g.dtype = a->dtype; g.act = a->act;
    g.M = a->m; g.N = a->n; g.K = a->k;
    g.sources = g.groups = 1;
    g.a[0] = mat(a->x, a->m, a->k, a->ldx, a->m > 0);
    g.b[0] = mat(a->w, a->n, a->k, a->ldw, true);
    g.bias[0] = mat.vec(a->bias);
    g.res = mat(a->res, a->m, a->n, a->ldres, false);
    g.out[0] = mat(a->y, a->m, a->n, a->ldy, a->m > 0);
    g.out[1] = mat(a->z, a->m, a->n, a->ldz, false);
    if (mat.rc) return mat.rc;
    if (shared({a->y, a->z}, {a->x, a->w, a->bias}) || (a->res && (a->z == a->res || (a->y == a->res && a->m > 1 && a->ldy != a->ldres)))) return DLF_E_INVALID_ARG;
    Steps steps{s, ask};
    const bool few = dense_gemv_takes(g);
    if (a->m == 0 || few) {
        if (only_workspace(ask, 0) || a->m == 0) return DLF_OK;
        rc = steps.begin();
        return rc ? rc : steps.gemv(g);
    }
    Carver carve{base_of(ws, ask)};
    Operands op{carve};
    g.a[0] = op(g.a[0], a->m, a->k);
    g.b[0] = op(g.b[0], a->n, a->k);
    if (only_workspace(ask, carve.used)) return DLF_OK;
    rc = ready(ask, ws, ws_bytes, carve.used, &steps);
    if (rc == DLF_OK) rc = steps.pack(op.jobs, op.n);
    return rc ? rc : steps.gemm(g);
}

int linear_grad(const dlf_linear_grad_args* a, void* ws, size_t ws_bytes, cudaStream_t s, Ask* ask) {
    if (!a) return DLF_E_INVALID_ARG;
    int rc = check_sizes(a->dtype, a->act, a->m, a->k, a->n);
    if (rc) return rc;
    const bool has_act = a->act != DLF_ACT_NONE, some = a->m > 0;
    Mats mat;
    const Mat dy = mat(a->dy, a->m, a->n, a->lddy, some), x = mat(a->x, a->m, a->k, a->ldx, some && a->dw);
    const Mat w = mat(a->w, a->n, a->k, a->ldw, some && a->dx), z = mat(a->z, a->m, a->n, a->ldz, some && has_act);
    const Mat dx = mat(a->dx, a->m, a->k, a->lddx, false), dw = mat(a->dw, a->n, a->k, a->lddw, false);
    const Mat dz_out = mat(a->dz, a->m, a->n, a->lddz, false);
    float* db = const_cast<float*>(mat.vec(a->db));
    if (mat.rc) return mat.rc;
    if (shared({a->dx, a->dw, a->db, a->dz}, {a->x, a->w}) || shared({a->dx, a->dw, a->db}, {a->dy, has_act ? a->z : nullptr})) return DLF_E_INVALID_ARG;
    if (some && a->m > 1 && a->dz && ((a->dz == a->dy && a->lddz != a->lddy) || (has_act && a->dz == a->z && a->lddz != a->ldz))) return DLF_E_INVALID_ARG;
    Steps steps{s, ask};
    if (!some) {
        if (only_workspace(ask, 0)) return DLF_OK;
        rc = steps.zero(dw, a->n, a->k);
        return rc ? rc : steps.zero(db, a->n);
    }
    Carver carve{base_of(ws, ask)};
    Operands op{carve};
    const Mat xo = dw.p ? op(x, a->m, a->k) : x, wo = dx.p ? op(w, a->n, a->k) : w;
    // dz, as the products read it: dy itself where nothing lies between, the caller's dz, or a matrix of its own.  16 bits wide, as the tensor
    // cores take their operands: half a step of each term, which leaves a sum of many terms 1.4 times as far from 64 bits as its own
    // last rounding does (bf16 2.35e-3 against 1.66e-3, fp16 2.93e-4 against 2.07e-4).  db sums what is not rounded yet.
    const bool products = dx.p || dw.p;
    Mat dz{nullptr, 0};
    if (products) dz = !has_act && dense_rows16(dy) ? dy : dz_out.p && dense_rows16(dz_out) ? dz_out : carve.matrix(a->m, a->n);
    if (only_workspace(ask, carve.used)) return DLF_OK;
    rc = ready(ask, ws, ws_bytes, carve.used, &steps);
    if (rc == DLF_OK) rc = steps.pack(op.jobs, op.n);
    if (rc) return rc;
    const bool own_dz = products && dz.p != dy.p;
    if (own_dz || dz_out.p || db) {
        DenseGrad d{};
        d.dtype = a->dtype; d.act = a->act;
        d.M = a->m; d.N = a->n;
        d.dy = dy; d.z = has_act ? z : Mat{nullptr, 0};
        if (own_dz) d.d0 = dz;
        if (dz_out.p && dz_out.p != d.d0.p) d.d0c = dz_out;
        d.db0 = db;
        rc = steps.grad(d);
        if (rc) return rc;
    }
    DenseGemm g[2] = {};
    int n = 0;
    if (dx.p) {   // dx[m][k] = sum over n of dz[m][n] w[n][k]
        DenseGemm& q = g[n++];
        q.dtype = a->dtype;
        q.sources = q.groups = 1;
        q.M = a->m; q.N = a->k; q.K = a->n;
        q.a[0] = dz; q.b[0] = wo; q.b_mn = true;
        q.out[0] = dx;
    }
    if (dw.p) {   // dw[n][k] = sum over m of dz[m][n] x[m][k]
        DenseGemm& q = g[n++];
        q.dtype = a->dtype;
        q.sources = q.groups = 1;
        q.M = a->n; q.N = a->k; q.K = a->m;
        q.a[0] = dz; q.b[0] = xo; q.a_mn = q.b_mn = true;
        q.out[0] = dw;
    }
    return steps.grads(g, n);
}

int gated(const dlf_gated_args* a, void* ws, size_t ws_bytes, cudaStream_t s, Ask* ask) {
    if (!a) return DLF_E_INVALID_ARG;
    int rc = check_sizes(a->dtype, a->act, a->m, a->k, a->n);
    if (rc) return rc;
    Mats mat;
    DenseGemm g{};
    g.dtype = a->dtype; g.act = a->act;
    g.M = a->m; g.N = a->n; g.K = a->k;
    g.sources = g.groups = 1;
    g.gated = true;
    g.a[0] = mat(a->x, a->m, a->k, a->ldx, a->m > 0);
    g.b[0] = mat(a->wg, a->n, a->k, a->ldwg, true);
    g.b[1] = mat(a->wu, a->n, a->k, a->ldwu, true);
    g.bias[0] = mat.vec(a->bg);
    g.bias[1] = mat.vec(a->bu);
    g.out[0] = mat(a->h, a->m, a->n, a->ldh, a->m > 0);
    g.out[1] = mat(a->g, a->m, a->n, a->ldg, false);
    g.out[2] = mat(a->u, a->m, a->n, a->ldu, false);
    if (mat.rc) return mat.rc;
    if (shared({a->h, a->g, a->u}, {a->x, a->wg, a->wu, a->bg, a->bu})) return DLF_E_INVALID_ARG;
    Steps steps{s, ask};
    const bool few = dense_gemv_takes(g);
    if (a->m == 0 || few) {
        if (only_workspace(ask, 0) || a->m == 0) return DLF_OK;
        rc = steps.begin();
        return rc ? rc : steps.gemv(g);
    }
    Carver carve{base_of(ws, ask)};
    Operands op{carve};
    g.a[0] = op(g.a[0], a->m, a->k);
    g.b[0] = op(g.b[0], a->n, a->k);
    g.b[1] = op(g.b[1], a->n, a->k);
    if (only_workspace(ask, carve.used)) return DLF_OK;
    rc = ready(ask, ws, ws_bytes, carve.used, &steps);
    if (rc == DLF_OK) rc = steps.pack(op.jobs, op.n);
    return rc ? rc : steps.gemm(g);
}

int gated_grad(const dlf_gated_grad_args* a, void* ws, size_t ws_bytes, cudaStream_t s, Ask* ask) {
    if (!a) return DLF_E_INVALID_ARG;
    int rc = check_sizes(a->dtype, a->act, a->m, a->k, a->n);
    if (rc) return rc;
    const bool some = a->m > 0, any_dw = a->dwg || a->dwu;
    Mats mat;
    DenseGrad d{};
    d.dtype = a->dtype; d.act = a->act;
    d.M = a->m; d.N = a->n;
    d.gated = true;
    d.dy = mat(a->dh, a->m, a->n, a->lddh, some);
    d.z = mat(a->g, a->m, a->n, a->ldg, some);
    d.u = mat(a->u, a->m, a->n, a->ldu, some);
    const Mat x = mat(a->x, a->m, a->k, a->ldx, some && any_dw);
    const Mat wg = mat(a->wg, a->n, a->k, a->ldwg, some && a->dx), wu = mat(a->wu, a->n, a->k, a->ldwu, some && a->dx);
    const Mat dx = mat(a->dx, a->m, a->k, a->lddx, false);
    const Mat dwg = mat(a->dwg, a->n, a->k, a->lddwg, false), dwu = mat(a->dwu, a->n, a->k, a->lddwu, false);
    d.db0 = const_cast<float*>(mat.vec(a->dbg));
    d.db1 = const_cast<float*>(mat.vec(a->dbu));
    if (mat.rc) return mat.rc;
    if (shared({a->dx, a->dwg, a->dwu, a->dbg, a->dbu}, {a->dh, a->x, a->wg, a->wu, a->g, a->u})) return DLF_E_INVALID_ARG;
    Steps steps{s, ask};
    if (!some) {
        if (only_workspace(ask, 0)) return DLF_OK;
        rc = steps.zero(dwg, a->n, a->k);
        if (!rc) rc = steps.zero(dwu, a->n, a->k);
        if (!rc) rc = steps.zero(d.db0, a->n);
        return rc ? rc : steps.zero(d.db1, a->n);
    }
    Carver carve{base_of(ws, ask)};
    Operands op{carve};
    const Mat xo = any_dw ? op(x, a->m, a->k) : x, wgo = dx.p ? op(wg, a->n, a->k) : wg, wuo = dx.p ? op(wu, a->n, a->k) : wu;
    // (dg and du are rounded once on their way into the products, as linear_grad's dz is)
    if (dx.p || dwg.p) d.d0 = carve.matrix(a->m, a->n);
    if (dx.p || dwu.p) d.d1 = carve.matrix(a->m, a->n);
    if (only_workspace(ask, carve.used)) return DLF_OK;
    rc = ready(ask, ws, ws_bytes, carve.used, &steps);
    if (rc == DLF_OK) rc = steps.pack(op.jobs, op.n);
    if (rc) return rc;
    rc = steps.grad(d);
    if (rc) return rc;
    DenseGemm g[2] = {};
    int n = 0;
    if (dx.p) {   // dx = dg wg + du wu, one sum
        DenseGemm& q = g[n++];
        q.dtype = a->dtype;
        q.sources = 2; q.groups = 1;
        q.M = a->m; q.N = a->k; q.K = a->n;
        q.a[0] = d.d0; q.a[1] = d.d1; q.b[0] = wgo; q.b[1] = wuo; q.b_mn = true;
        q.out[0] = dx;
    }
    if (any_dw) {   // dwg = dg^T x and dwu = du^T x, two groups of tiles
        DenseGemm& q = g[n++];
        q.dtype = a->dtype;
        q.sources = 1; q.groups = dwg.p && dwu.p ? 2 : 1;
        q.M = a->n; q.N = a->k; q.K = a->m;
        q.a[0] = dwg.p ? d.d0 : d.d1; q.b[0] = xo; q.a_mn = q.b_mn = true;
        q.out[0] = dwg.p ? dwg : dwu;
        if (q.groups > 1) {
            q.a[1] = d.d1;
            q.out[1] = dwu;
        }
    }
    return steps.grads(g, n);
}

}  // namespace

int launch_dense_pack(const DensePack* jobs, int n, int sms, cudaStream_t s) {
    PackParams p{};
    p.n = n;
    for (int i = 0; i < n; i++) {
        p.job[i] = jobs[i];
        p.first[i + 1] = p.first[i] + jobs[i].rows * ceil_div(jobs[i].cols, 8);
    }
    const int grid = static_cast<int>(std::min<int64_t>(ceil_div(p.first[n], 256), 8ll * sms));
    const cudaError_t e = launch_kernel(p.first[n] < (1ll << 31) - (1ll << 24) ? dense_pack_kernel<uint32_t> : dense_pack_kernel<uint64_t>, grid, 256, 0, s, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

int launch_dense_grad(const DenseGrad& g, int sms, cudaStream_t s) {
    const GradLayout l = grad_layout(g, sms);
    GradFn fn = nullptr;
    if (g.dtype == DLF_BF16) fn = l.v8 ? pick_grad<__nv_bfloat16, 8>(g.gated, l.wide, g.act) : pick_grad<__nv_bfloat16, 2>(g.gated, l.wide, g.act);
    else fn = l.v8 ? pick_grad<__half, 8>(g.gated, l.wide, g.act) : pick_grad<__half, 2>(g.gated, l.wide, g.act);
    const cudaError_t e = launch_kernel(fn, l.grid, kGradThreads, 0, s, g);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}

}  // namespace dlf

extern "C" {

int dlf_dense_sync(void* stream) {
    static thread_local int told[dlf::kMaxDevices][2];   // what this thread has been told of
    const int dev = dlf::current_device_slot();
    if (dev < 0) return DLF_E_UNSUPPORTED;
    int now[2] = {0, 0};
    int rc = dlf::dense_pair_gave_up(static_cast<cudaStream_t>(stream), &now[0]);
    if (rc == DLF_OK) rc = dlf::dense_lat_gave_up(static_cast<cudaStream_t>(stream), &now[1]);
    if (rc) return rc;
    const bool more = now[0] != told[dev][0] || now[1] != told[dev][1];
    told[dev][0] = now[0];
    told[dev][1] = now[1];
    return more ? DLF_E_TIMEOUT : DLF_OK;
}

int dlf_dense_debug_stall(int which, int limit_us, void* stream) {
    if ((which != 0 && which != 1) || limit_us < 1 || limit_us > 1000000) return DLF_E_INVALID_ARG;
    const unsigned long long ns = static_cast<unsigned long long>(limit_us) * 1000;
    return which ? dlf::dense_lat_stall(ns, static_cast<cudaStream_t>(stream)) : dlf::dense_pair_stall(ns, static_cast<cudaStream_t>(stream));
}

// What a call would do: its workspace, its kernels.
#define DLF_DENSE_ENTRIES(OP)                                                                                                  \
    int dlf_##OP##_workspace_bytes(const dlf_##OP##_args* a, size_t* bytes) {                                                   \
        if (!bytes) return DLF_E_INVALID_ARG;                                                                                   \
        dlf::Ask ask{bytes, nullptr, 0, 0, 0};                                                                                  \
        return dlf::OP(a, nullptr, 0, nullptr, &ask);                                                                           \
    }                                                                                                                           \
    int dlf_##OP##_kernels(const dlf_##OP##_args* a, int sm_count, char* text, size_t bytes) {                                  \
        if (!text || bytes == 0 || sm_count < 0) return DLF_E_INVALID_ARG;                                                      \
        text[0] = 0;                                                                                                            \
        dlf::Ask ask{nullptr, text, bytes, 0, sm_count};                                                                        \
        return dlf::OP(a, nullptr, 0, nullptr, &ask);                                                                           \
    }                                                                                                                           \
    int dlf_##OP(const dlf_##OP##_args* a, void* workspace_dev, size_t bytes, void* stream) {                                   \
        return dlf::OP(a, workspace_dev, bytes, static_cast<cudaStream_t>(stream), nullptr);                                    \
    }
DLF_DENSE_ENTRIES(linear)
DLF_DENSE_ENTRIES(linear_grad)
DLF_DENSE_ENTRIES(gated)
DLF_DENSE_ENTRIES(gated_grad)
#undef DLF_DENSE_ENTRIES

}  // extern "C"
