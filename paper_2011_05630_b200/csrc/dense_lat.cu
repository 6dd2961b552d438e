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
constexpr int kProdWarp0 = kEpiWarps, kProdWarps = 3;   // behind the first round of the ring warp w loads stages w, w + 3, ...
constexpr int kMmaWarp = kProdWarp0 + kProdWarps, kMmaWarps = 2;   // issuers: warp w takes chunks w, w + 2, ...
constexpr int kThreads = 32 * (kMmaWarp + kMmaWarps);
constexpr int kMaxBN = 128, kMaxStages = 12;
constexpr int kMaxDynSmem = 225 * 1024;
constexpr int kPairSmem = 110 * 1024;        // two CTAs fit an SM: one's set-up and last rows behind the other's products
constexpr int kAloneSmem = 200 * 1024;       // more than this leaves no room for another tensor-core kernel's CTA on the SM
enum { EPI_PLAIN = 0, EPI_LINEAR = 1, EPI_GATED = 2 };

// One product, or the two gradients' products that share a launch.
struct LatJob {
    CUtensorMap a[2], b[2];
    Mat o[3];
    long long M, N, group_tiles;
    int tiles_n, rows;                 // rows: of A in a tile
    int chunks1, total, share;         // 64-value chunks of K: of the first source, of both, of a CTA
    int stages, a_bytes, stage_bytes, red_off, rows_per;
    int groups;
    bool amn, vec;                     // vec: every row that is read or written here starts on a 16-byte boundary
};
template <int JOBS>
struct LatParams {
    LatJob job[JOBS];
    Mat res;
    const float* bias[2];
    int act, BN, first1;               // first1: CTAs of the first job
};

// From the sums of W (an even number) outputs of a row to what is stored: v (and u of a gated tile), the biases, what is added.
template <int EPI, int W, typename PUT>
__device__ __forceinline__ void finish(int act_code, float (&v)[W], float (&u)[W], const float (&r)[W], PUT&& put) {
    if (EPI == EPI_LINEAR) {
#pragma unroll
        for (int i = 0; i < W; i++) v[i] += r[i];
    }
    if (EPI != EPI_PLAIN) put(1, v);
    if (EPI == EPI_GATED) put(2, u);
    if (EPI != EPI_PLAIN)
        with_act(act_code, [&](auto act) {
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                float2 a = act2<act.value>(make_float2(v[i], v[i + 1]));
                if (EPI == EPI_GATED) a = mul2(a, make_float2(u[i], u[i + 1]));
                v[i] = a.x; v[i + 1] = a.y;
            }
        });
    put(0, v);
}

template <typename T, int EPI, int SPLIT>
__global__ void __cluster_dims__(SPLIT, 1, 1) __launch_bounds__(kThreads, SPLIT == 1 ? 2 : 1) dense_lat_kernel(const __grid_constant__ LatParams<EPI == EPI_PLAIN ? 2 : 1> P) {
    constexpr bool BMN = EPI == EPI_PLAIN;   // (a forward product's operands lie along K; of the gradients' B lies across, and A, too, for weights)
    const bool job1 = EPI == EPI_PLAIN && static_cast<int>(blockIdx.x) >= P.first1;
    const LatJob& p = P.job[EPI == EPI_PLAIN && job1 ? 1 : 0];
    const bool amn = EPI == EPI_PLAIN && p.amn;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], tfull_bar, red_bar;
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s, red_abort_s;
    __shared__ float bias_s[kMaxBN];

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sbase = smem_raw + (base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &abort_s;
    int* status = g_dense_status;
    const int rank = SPLIT > 1 ? static_cast<int>(cluster_rank()) : 0;
    long long tile = (static_cast<int>(blockIdx.x) - (job1 ? P.first1 : 0)) / SPLIT;
    const int group = p.groups > 1 && tile >= p.group_tiles ? 1 : 0;
    tile -= group ? p.group_tiles : 0;
    const long long tm = tile / p.tiles_n;
    const long long n0 = (tile - tm * p.tiles_n) * (EPI == EPI_GATED ? P.BN / 2 : P.BN), m0 = tm * p.rows;
    const int k_first = rank * p.share, k_count = min(p.share, p.total - k_first);
    const int live = static_cast<int>(min(static_cast<long long>(p.rows), p.M - m0));   // rows of the tile that exist

    // A stage's boxes, those of A first: where each comes from and goes to.  (Worked out once: with the choices in the loop the pairs' weight
    // gradients took 5 % longer.)
    const int boxes_a = amn ? 2 : 1, boxes = boxes_a + (EPI == EPI_GATED ? 2 : BMN ? P.BN / 64 : 1);
    const uint32_t stage_tx = static_cast<uint32_t>(p.a_bytes + P.BN * 128);
    struct Box {
        const CUtensorMap *map0, *map1;   // of the first source and of the second
        int off, row;
        bool across;
    };
    auto box_of = [&](int bx) {
        const int j = bx - boxes_a;
        Box b;
        if (j < 0) {
            b = Box{&p.a[group], &p.a[1], bx * 8192, static_cast<int>(m0) + bx * 64, amn};
        } else {
            b.map0 = &p.b[EPI == EPI_GATED ? j : 0];
            b.map1 = &p.b[1];
            b.off = p.a_bytes + (EPI == EPI_GATED ? j * P.BN * 64 : j * 8192);
            b.row = static_cast<int>(n0) + (BMN ? j * 64 : 0);
            b.across = BMN;
        }
        return b;
    };
    auto load_box = [&](const Box& b, int i, int st) {   // of chunk i of this CTA's share into stage st
        const int c = k_first + i;
        const bool second = c >= p.chunks1;
        const int k0 = (second ? c - p.chunks1 : c) * 64;
        tma_load_2d(sbase + st * p.stage_bytes + b.off, second ? b.map1 : b.map0, &full_bar[st], b.across ? b.row : k0, b.across ? k0 : b.row);
    };
    if (warp == kProdWarp0) {
        if (lane < kMaxStages) {
            mbar_init(&full_bar[lane], 1);
            mbar_init(&empty_bar[lane], 1);
        }
        if (lane == 0) {
            abort_s = 0;
            red_abort_s = 0;
            mbar_init(&tfull_bar, kMmaWarps);
            mbar_init(&red_bar, 1);
        }
        fence_barrier_init();
        // the bytes that the cluster's CTAs will send here (before the cluster's barrier, which every sender waits for)
        if (SPLIT > 1 && lane == 0) mbar_expect_tx(&red_bar, static_cast<uint32_t>(SPLIT * max(0, min(p.rows_per, live - rank * p.rows_per)) * P.BN) * 4u);
        __syncwarp();
        // the ring's first round is on its way before the rest of the set-up (a lane a stage)
        pdl_wait();
        if (lane < min(p.stages, k_count)) {
            mbar_expect_tx(&full_bar[lane], stage_tx);
#pragma unroll 1
            for (int bx = 0; bx < boxes; bx++) load_box(box_of(bx), lane, lane);
        }
        __syncwarp();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&tmem_base_s, kMaxBN * kMmaWarps);
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
        // ---- producers: lane i issues a stage's i-th box ----
        const int w = warp - kProdWarp0;
        const Box mine = box_of(min(lane, boxes - 1));
        int turn = 0, st = 0;
        uint32_t ph = 0;
#pragma unroll 1
        for (int i = p.stages; i < k_count; i++) {
            if (turn == w) {
                if (!mbar_wait_warp<true>(&empty_bar[st], ph, abort_flag, status, 0xA00 | (blockIdx.x << 12))) break;
                if (lane == 0) mbar_expect_tx(&full_bar[st], stage_tx);
                __syncwarp();
                if (lane < boxes) load_box(mine, i, st);
                __syncwarp();
            }
            if (++turn == kProdWarps) turn = 0;
            if (++st == p.stages) { st = 0; turn = 0; ph ^= 1u; }
        }
    } else if (warp >= kMmaWarp) {
        // ---- issuers.  A run of matrix instructions holds its warp until it has almost executed, and what the warp does between two
        // runs takes as long again: two warps with an accumulator each hide one behind the other (550 -> 300 clocks a chunk);
        // the epilogue adds the two sums ----
        const int w = warp - kMmaWarp;
        const uint32_t d_tmem = tmem_base + w * kMaxBN;
        const int last = k_count - 1 - ((k_count - 1 - w) & 1);   // this issuer's last chunk (negative: it has none)
        const uint32_t b0 = BMN ? umma_desc_mn_lo(base + p.a_bytes, 8192) : umma_desc_lo(base + p.a_bytes);
        const uint32_t stage16 = static_cast<uint32_t>(p.stage_bytes) >> 4;
        int st = w % p.stages;
        uint32_t ph = static_cast<uint32_t>(w / p.stages) & 1u, off = static_cast<uint32_t>(st) * stage16;
        auto multiply = [&](auto across) {   // (a loop for each kind of operand A: its steps are constants)
            constexpr bool AMN = across.value;
            const uint32_t idesc = dense_idesc<T>(128, 0, AMN, BMN) | (static_cast<uint32_t>(P.BN >> 3) << 17);
            const uint32_t a0 = AMN ? umma_desc_mn_lo(base, 8192) : umma_desc_lo(base);
#pragma unroll 1
            for (int i = w; i < k_count; i += 2) {
                if (!mbar_wait_warp<true>(&full_bar[st], ph, abort_flag, status, 0xA10 | (blockIdx.x << 12))) break;
                tc_fence_after_sync();
                if (elect_one()) {
                    umma_chunk<1, AMN, BMN>(d_tmem, a0 + off, b0 + off, idesc, i != w);
                    if (i + p.stages < k_count) umma_commit(&empty_bar[st]);
                    if (i == last) umma_commit(&tfull_bar);
                }
                __syncwarp();
                st += 2;
                off += 2 * stage16;
                if (st >= p.stages) { st -= p.stages; ph ^= 1u; off -= static_cast<uint32_t>(p.stages) * stage16; }
            }
        };
        if (amn) multiply(std::integral_constant<bool, EPI == EPI_PLAIN>{});
        else multiply(std::false_type{});
        if (last < 0 && lane == 0) mbar_arrive(&tfull_bar);
    } else {
        // ---- epilogue: the sums go to shared memory (of the CTA that finishes them), row by row, and from there in runs of 8 outputs
        // that lie side by side in memory ----
        const int q = warp & 3, half = warp >> 2, m = q * 32 + lane;
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        const int out_bn = EPI == EPI_GATED ? P.BN / 2 : P.BN;
        const int my_rows = max(0, min(p.rows_per, live - rank * p.rows_per)), runs = p.vec ? out_bn / 8 : out_bn / 8 + 1;   // (of 8 outputs in a row: below)
        const uint32_t by_runs = 65536u / static_cast<uint32_t>(runs) + 1u;                                 // i / runs for the at most 2176 runs of a tile
        const long long row_first = m0 + rank * p.rows_per;
        const int n_cols = static_cast<int>(min(static_cast<long long>(out_bn), p.N - n0));
        if (EPI != EPI_PLAIN && threadIdx.x < P.BN) {
            const int c = EPI == EPI_GATED && static_cast<int>(threadIdx.x) >= out_bn ? static_cast<int>(threadIdx.x) - out_bn : static_cast<int>(threadIdx.x);
            const float* b = P.bias[EPI == EPI_GATED && static_cast<int>(threadIdx.x) >= out_bn ? 1 : 0];
            bias_s[threadIdx.x] = b && c < n_cols ? ld_map(b + n0 + c) : 0.0f;
        }
        // A run is 8 outputs that are a piece of 16 bytes in memory: where rows start off the 16-byte boundaries, a row's first and
        // last runs are not whole.  Run i of this CTA: row and first column (of n_cols), negative behind the last run.
        const int total = my_rows * runs;
        const unsigned short* const out0 = static_cast<const unsigned short*>(p.o[EPI == EPI_PLAIN ? group : 0].p) + row_first * p.o[EPI == EPI_PLAIN ? group : 0].ld + n0;
        const int64_t out_ld = p.o[EPI == EPI_PLAIN ? group : 0].ld;
        auto run_at = [&](auto vec, int i, int* c) {
            if (i >= total) return -1;
            const int r = static_cast<int>(static_cast<uint32_t>(i) * by_runs >> 16);
            *c = (i - r * runs) * 8;
            if (vec.value) return *c < n_cols ? r : -1;
            *c -= static_cast<int>((reinterpret_cast<uintptr_t>(out0 + r * out_ld) >> 1) & 7);
            return *c < n_cols && *c + 8 > 0 ? r : -1;
        };
        // 8 values of a row from column c on, those that exist
        auto fetch8 = [&](auto vec, const unsigned short* q, int c) {
            if (vec.value ? c + 8 <= n_cols : c >= 0 && c + 8 <= n_cols && (reinterpret_cast<uintptr_t>(q) & 15) == 0) return ld_map(reinterpret_cast<const uint4*>(q));
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int d = c + 2 * e;
                w[e] = (d >= 0 && d < n_cols ? ld_map(q + 2 * e) : 0u) | (d + 1 >= 0 && d + 1 < n_cols ? static_cast<uint32_t>(ld_map(q + 2 * e + 1)) : 0u) << 16;
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
        };
        // what a thread's next runs have to add is fetched kItems runs at a time, the first ones behind the products
        constexpr int kItems = 4;
        const bool add = EPI == EPI_LINEAR && P.res.p != nullptr;
        uint4 res[kItems] = {};
        auto fetch_res = [&](auto vec, int i0) {
#pragma unroll
            for (int it = 0; it < kItems; it++) {
                int c = 0;
                const int r = run_at(vec, i0 + it * 32 * kEpiWarps, &c);
                res[it] = make_uint4(0u, 0u, 0u, 0u);
                if (add && r >= 0) res[it] = fetch8(vec, static_cast<const unsigned short*>(P.res.p) + (row_first + r) * P.res.ld + n0 + c, c);
            }
        };
        if (add && p.vec) fetch_res(std::true_type{}, threadIdx.x);
        else if (add) fetch_res(std::false_type{}, threadIdx.x);
        bool ok = mbar_wait_warp<true>(&tfull_bar, 0u, abort_flag, status, 0xA20 | (blockIdx.x << 12));
        tc_fence_after_sync();
        const int dest = SPLIT > 1 ? min(m / p.rows_per, SPLIT - 1) : 0, row = m - dest * p.rows_per;
        const uint32_t slab = static_cast<uint32_t>(p.rows_per * P.BN * 4);   // one rank's partial rows
        // (a row's 16-byte vectors are stored in an order that depends on the row: the lanes of a warp fall into different banks)
        const uint32_t swz = static_cast<uint32_t>(row) & 7u;
        uint32_t dst = base + p.red_off + rank * slab + row * P.BN * 4, dst_bar = 0;
        if (SPLIT > 1) {
            dst = mapa(dst, dest);
            dst_bar = mapa(smem_u32(&red_bar), dest);
            cluster_wait();   // every CTA of the cluster runs and its barrier expects these rows
        }
#pragma unroll 1
        for (int c0 = half * 16; c0 < P.BN; c0 += 32) {
            uint32_t r0[16], r1[16];
            float v[16];
            tmem_ld16_issue(taddr + c0, r0);
            tmem_ld16_issue(taddr + kMaxBN + c0, r1);
            tmem_ld16_wait(r0);
            tmem_ld16_wait(r1);
#pragma unroll
            for (int e = 0; e < 16; e++) v[e] = k_count > 1 ? __uint_as_float(r0[e]) + __uint_as_float(r1[e]) : __uint_as_float(r0[e]);
            if (m < live) {   // (sent whatever happened: the other CTAs wait for the bytes)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t at = dst + ((static_cast<uint32_t>((c0 >> 2) + e) ^ swz) << 4);
                    if (SPLIT > 1) st_async_v4(at, v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3], dst_bar);
                    else *reinterpret_cast<float4*>(sbase + (at - base)) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                }
            }
            __syncwarp();
        }
        // All rows of this CTA are here.  It must not retire before that, whatever its own part came to, hence a limit above
        // the senders' and a flag of its own.
        if (SPLIT > 1) ok = mbar_wait<true>(&red_bar, 0u, &red_abort_s, status, 0xA30 | (blockIdx.x << 12), 4 * kWaitLimitNs) && ok;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");   // (the biases; with one CTA the sums)
        const uint8_t* red = sbase + p.red_off;
        auto finish_runs = [&](auto vec) {
#pragma unroll 1
            for (int i0 = threadIdx.x; i0 < total; i0 += kItems * 32 * kEpiWarps) {
                if (add && i0 != static_cast<int>(threadIdx.x)) fetch_res(vec, i0);
#pragma unroll
                for (int it = 0; it < kItems; it++) {
                    int c = 0;
                    const int r = run_at(vec, i0 + it * 32 * kEpiWarps, &c);
                    if (r < 0) continue;
                    float v[8], u[8], a[8];
                    auto sum = [&](int col, float (&s)[8]) {
                        const uint8_t* const at = red + r * P.BN * 4;
                        const uint32_t swap = static_cast<uint32_t>(r) & 7u;
#pragma unroll
                        for (int e = 0; e < 8; e++) s[e] = 0.0f;
                        if (vec.value) {
                            const uint32_t x16 = (static_cast<uint32_t>(col >> 2) ^ swap) << 4;
#pragma unroll
                            for (int sp = 0; sp < SPLIT; sp++) {
                                const float4 x = *reinterpret_cast<const float4*>(at + sp * slab + x16), y = *reinterpret_cast<const float4*>(at + sp * slab + (x16 ^ 16u));
                                s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
                                s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; e++) {
                                const int d = min(max(col + e, 0), P.BN - 1);   // (a column that does not exist: any value)
                                const uint8_t* const q = at + (((static_cast<uint32_t>(d) >> 2) ^ swap) << 4) + (d & 3) * 4;
#pragma unroll
                                for (int sp = 0; sp < SPLIT; sp++) s[e] += *reinterpret_cast<const float*>(q + sp * slab);
                            }
                        }
                        if (EPI != EPI_PLAIN) {
#pragma unroll
                            for (int e = 0; e < 8; e++) s[e] += bias_s[vec.value ? col + e : min(max(col + e, 0), P.BN - 1)];
                        }
                    };
                    sum(c, v);
                    if (EPI == EPI_GATED) sum(out_bn + c, u);
                    const T* in = reinterpret_cast<const T*>(&res[it]);
#pragma unroll
                    for (int e = 0; e < 8; e++) a[e] = add ? to_f32(in[e]) : 0.0f;
                    finish<EPI>(P.act, v, u, a, [&](int which, const float(&f)[8]) {
                        const Mat& o = p.o[EPI == EPI_PLAIN ? group : which];
                        if (!o.p) return;
                        T* t = static_cast<T*>(const_cast<void*>(o.p)) + (row_first + r) * o.ld + n0 + c;
                        if (vec.value ? c + 8 <= n_cols : c >= 0 && c + 8 <= n_cols && (reinterpret_cast<uintptr_t>(t) & 15) == 0) {
                            *reinterpret_cast<uint4*>(t) = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; e++)
                                if (c + e >= 0 && c + e < n_cols) t[e] = from_f32<T>(f[e]);
                        }
                    });
                }
            }
        };
        if (ok && p.vec) finish_runs(std::true_type{});
        else if (ok) finish_runs(std::false_type{});
        tc_fence_before_sync();
    }
    __syncwarp();
    if (SPLIT > 1 && warp >= kEpiWarps) cluster_wait();
    __syncthreads();
    if (warp == kMmaWarp) {
        if (lane == 0 && (abort_s || red_abort_s)) dense_count_abort();
        if (abort_s) __nanosleep(20000);   // let copies in flight land before the CTA retires
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, kMaxBN * kMmaWarps);
    }
}

// The layout of a tile in shared memory: ring depth, and where the cluster's partial sums go.
bool lay_out(const DenseGemm& g, const DenseLatChoice& c, LatJob* p, size_t* smem) {
    p->rows = g.a_mn ? static_cast<int>(std::min<int64_t>(g.M, 128)) : static_cast<int>((g.M + (g.M + 127) / 128 - 1) / ((g.M + 127) / 128));
    p->a_bytes = g.a_mn ? 16384 : (p->rows + 7) / 8 * 1024;
    p->stage_bytes = p->a_bytes + c.bn * 128;
    p->chunks1 = static_cast<int>((g.K + 63) / 64);
    p->total = p->chunks1 * g.sources;
    p->share = (p->total + c.split - 1) / c.split;
    p->rows_per = (p->rows + c.split - 1) / c.split;
    if (c.split > 1 && (c.split - 1) * p->share >= p->total) return false;   // (a CTA without work)
    const int red = c.split > 1 ? c.split * p->rows_per * c.bn * 4 : 0;
    const int slack = 16384 - p->a_bytes;   // the tensor core reads 128 rows of A, behind the ring's last ones too: memory of this CTA all the same
    for (int budget : {kPairSmem, kMaxDynSmem}) {
        if ((c.split > 1 || c.deep) && budget == kPairSmem) continue;
        p->stages = std::min({kMaxStages, (budget - 1024 - red - slack) / p->stage_bytes, p->share});
        if (p->stages < p->share) p->stages &= ~1;   // the ring goes round: a stage belongs to one issuer
        if (p->stages >= std::min(p->share, 4)) break;
    }
    if (p->stages < std::min(p->share, 3)) return false;
    const int ring = p->stages * p->stage_bytes + slack;
    p->red_off = c.split > 1 ? ring : 0;   // (alone, a CTA's sums go where the ring was)
    *smem = static_cast<size_t>(std::max(ring + red, p->red_off + c.split * p->rows_per * c.bn * 4)) + 1024;
    if (c.split > 1) *smem = std::max<size_t>(*smem, kAloneSmem);
    return true;
}

int fill_job(const DenseGemm& g, const DenseLatChoice& c, LatJob* p, size_t* smem) {
    size_t mine = 0;
    if (!lay_out(g, c, p, &mine)) return DLF_E_UNSUPPORTED;
    *smem = std::max(*smem, mine);
    for (int i = 0; i < 2; i++) {
        const Mat &a = g.a[i], &b = g.b[i];
        int rc = DLF_OK;
        if (a.p) rc = g.a_mn ? dense_map(&p->a[i], a, g.K, g.M, 64, 64) : dense_map(&p->a[i], a, g.M, g.K, p->a_bytes / 128, 64);
        if (b.p && rc == DLF_OK) rc = g.b_mn ? dense_map(&p->b[i], b, g.K, g.N, 64, 64) : dense_map(&p->b[i], b, g.N, g.K, g.gated ? c.bn / 2 : c.bn, 64);
        if (rc) return rc;
    }
    for (int i = 0; i < 3; i++) p->o[i] = g.out[i];
    p->vec = dense_rows16(g.res) && dense_rows16(g.out[0]) && dense_rows16(g.out[1]) && dense_rows16(g.out[2]);
    p->M = g.M; p->N = g.N;
    const int step = g.gated ? c.bn / 2 : c.bn;
    p->tiles_n = static_cast<int>((g.N + step - 1) / step);
    p->group_tiles = (g.M + p->rows - 1) / p->rows * p->tiles_n;
    p->groups = g.groups;
    p->amn = g.a_mn;
    return DLF_OK;
}
template <typename FN, typename PARAMS>
int launch_lat(FN fn, const PARAMS& p, int grid, size_t smem, cudaStream_t s) {
    const int rc = dense_smem_attr(reinterpret_cast<const void*>(fn), kMaxDynSmem);
    if (rc) return rc;
    const cudaError_t e = launch_kernel(fn, grid, kThreads, smem, s, p);
    return e == cudaSuccess ? DLF_OK : cuda_fail(e);
}
template <typename T, int EPI, typename PARAMS>
int launch_split(int split, const PARAMS& p, int grid, size_t smem, cudaStream_t s) {
    switch (split) {
        case 1: return launch_lat(dense_lat_kernel<T, EPI, 1>, p, grid, smem, s);
        case 2: return launch_lat(dense_lat_kernel<T, EPI, 2>, p, grid, smem, s);
        case 4: return launch_lat(dense_lat_kernel<T, EPI, 4>, p, grid, smem, s);
        default: return launch_lat(dense_lat_kernel<T, EPI, 8>, p, grid, smem, s);
    }
}

}  // namespace

bool dense_lat_possible(const DenseGemm& g, const DenseLatChoice& c, int* rows, int* stages, bool* two) {
    LatJob p;
    size_t smem;
    if (!lay_out(g, c, &p, &smem)) return false;
    *rows = p.rows;
    *stages = p.stages;
    *two = smem <= static_cast<size_t>(kPairSmem) + 2048;
    return true;
}

int launch_dense_lat(const DenseGemm* g, int n, const DenseLatChoice& c, cudaStream_t s) {
    const bool bf = g[0].dtype == DLF_BF16;
    size_t smem = 0;
    if (!g[0].b_mn) {
        LatParams<1> p;
        std::memset(&p, 0, sizeof(p));
        const int rc = fill_job(g[0], c, &p.job[0], &smem);
        if (rc) return rc;
        p.res = g[0].res;
        p.bias[0] = g[0].bias[0]; p.bias[1] = g[0].bias[1];
        p.act = g[0].act;
        p.BN = c.bn;
        const int grid = static_cast<int>(p.job[0].group_tiles * c.split);
        if (g[0].gated) return bf ? launch_split<__nv_bfloat16, EPI_GATED>(c.split, p, grid, smem, s) : launch_split<__half, EPI_GATED>(c.split, p, grid, smem, s);
        return bf ? launch_split<__nv_bfloat16, EPI_LINEAR>(c.split, p, grid, smem, s) : launch_split<__half, EPI_LINEAR>(c.split, p, grid, smem, s);
    }
    LatParams<2> p;
    std::memset(&p, 0, sizeof(p));
    p.BN = c.bn;
    int grid = 0;
    for (int i = 0; i < n; i++) {
        const int rc = fill_job(g[i], c, &p.job[i], &smem);
        if (rc) return rc;
        if (i == 1) p.first1 = grid;
        grid += static_cast<int>(p.job[i].group_tiles * g[i].groups * c.split);
    }
    if (n == 1) p.first1 = grid;
    return bf ? launch_split<__nv_bfloat16, EPI_PLAIN>(c.split, p, grid, smem, s) : launch_split<__half, EPI_PLAIN>(c.split, p, grid, smem, s);
}

int dense_lat_gave_up(cudaStream_t s, int* count) { return dense_gave_up(s, count); }
int dense_lat_stall(unsigned long long limit_ns, cudaStream_t s) { return dense_stall(limit_ns, s); }

}  // namespace dlf
